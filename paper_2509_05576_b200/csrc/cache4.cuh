// A key-value cache held in 4 bits: where its tokens go, writing and reading it, and attention of a few rows over it.
//
// Grid: every 32 values of a key or value share a min-max grid with 0 in its range, as the rows of a weight matrix do
// (ptq_minmax_grid).  Its step s is rounded UP to a number of 6 significant bits, so that s (c - z) with 4-bit codes has at most ten
// and is exactly an fp16 number: what the tensor cores multiply is what the cache stands for, and no product rounds an operand.
// Step and zero code share 16 bits: the fp16 pattern of s, whose low five bits are zero, with z in the lowest four.
//
// Layout: pages[page][kv_head][tile of 16 tokens][K codes | K grids | V codes | V grids], so that one tile of one head is one
// contiguous piece (2304 bytes for heads of 128) and comes in one bulk copy.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "fp8.cuh"
#include "tc.cuh"
#include <type_traits>

namespace ptq {

constexpr int kC4Tile = 16, kC4Group = 32;
constexpr float kC4MinStep = 1.9073486328125e-06f, kC4MaxStep = 2112.0f;     // 2^-19; 33 2^6: (16 + z) s and 16 s stay below 65504

__host__ __device__ constexpr int c4_side_bytes(int dim) { return kC4Tile * (dim / 2 + dim / kC4Group * 2); }
__host__ __device__ constexpr int c4_tile_bytes(int dim) { return 2 * c4_side_bytes(dim); }

struct Cache4 {
    uint8_t* pages;
    int num_pages, page_shift, kv_heads;       // page size = 1 << page_shift
};
template <int HD>
__device__ __forceinline__ uint8_t* c4_tile(const Cache4& c, int page, int head, int tile) {
    const int per = 1 << (c.page_shift - 4);
    return c.pages + (((int64_t)page * c.kv_heads + head) * per + tile) * c4_tile_bytes(HD);
}

// ------------------------------------------------------------------------------------------------------------
// Block tables and slots
// ------------------------------------------------------------------------------------------------------------
struct CachePlan {
    const int32_t* lens;          // [batch] tokens cached before
    const int32_t* fresh;         // [batch] new tokens
    int batch;
    int32_t* table;               // [batch][max_pages], in/out
    int64_t ldt;
    int max_pages;
    const int32_t* free_pages;
    int num_free, page_shift;
    int32_t* slots;               // [max_tokens]
    int32_t* positions;           // [max_tokens]
    int max_tokens;
    int32_t* cu;                  // [batch + 1]
    int32_t* lens_out;            // [batch]
    int32_t* taken;               // [1]
    int32_t* status;
};

constexpr int kPlanThreads = 1024, kPlanTokens = 4096;       // threads a CTA; tokens a CTA answers for

// Sums of (tokens, pages) over the CTA's threads before this one; totals in `all`.  One pair in 64 bits: tokens may reach 2^31
// (checked in 64 bits by the caller), so the two are scanned apart.
__device__ __forceinline__ longlong2 plan_scan(longlong2 v, longlong2* warp_sums, longlong2& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    longlong2 x = v;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, x.x, s), b = __shfl_up_sync(0xffffffffu, x.y, s);
        if (lane >= s) { x.x += a; x.y += b; }
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        longlong2 w = warp_sums[lane];
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) {
            const long long a = __shfl_up_sync(0xffffffffu, w.x, s), b = __shfl_up_sync(0xffffffffu, w.y, s);
            if (lane >= s) { w.x += a; w.y += b; }
        }
        warp_sums[lane] = w;
    }
    __syncthreads();
    all = warp_sums[31];
    const longlong2 before = warp ? warp_sums[warp - 1] : make_longlong2(0, 0);
    return make_longlong2(before.x + x.x - v.x, before.y + x.y - v.y);
}

// One launch.  Every CTA scans all requests (a thousand at a time) and answers for kPlanTokens tokens, four a thread, each of which
// finds its request by bisection; the first CTA also writes what belongs to requests.  Nothing is written before the whole batch is
// known to fit: a batch that does not leaves every slot at -1, no rows (cu = 0), the lengths as they were and the table untouched.
// A new page's first token is always new, so that the token writes the page's table entry.
struct PlanRequest { int len, n, have, want; bool ok; };
__device__ __forceinline__ PlanRequest plan_request(const CachePlan& p, int b) {
    PlanRequest r{0, 0, 0, 0, true};
    if (b >= p.batch) return r;
    const int ps = 1 << p.page_shift;
    r.len = p.lens[b];
    r.n = p.fresh[b];
    if (r.len < 0 || r.n < 0 || (long long)r.len + r.n > 0x7fffffffll - ps) return PlanRequest{0, 0, 0, 0, false};
    r.have = (r.len + ps - 1) >> p.page_shift;
    r.want = (r.len + r.n + ps - 1) >> p.page_shift;
    r.ok = r.want <= p.max_pages;
    return r;
}

__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(CachePlan p) {
    chained_begin();
    __shared__ longlong2 warp_sums[32];
    __shared__ int bad_request;
    __shared__ int at_token[kPlanThreads], at_page[kPlanThreads], at_len[kPlanThreads], at_have[kPlanThreads];
    const int ps = 1 << p.page_shift;
    const long long t0 = (long long)blockIdx.x * kPlanTokens, t1 = min(t0 + kPlanTokens, (long long)p.max_tokens);
    if (threadIdx.x == 0) bad_request = 0x7fffffff;
    __syncthreads();
    long long tokens = 0, pages = 0;
    PlanRequest r;
    longlong2 at, all;
    for (int first = 0; first < p.batch; first += kPlanThreads) {
        const int b = first + threadIdx.x;
        r = plan_request(p, b);
        at = plan_scan(make_longlong2(r.n, r.want - r.have), warp_sums, all);
        if (!r.ok || (b < p.batch && (tokens + at.x + r.n > p.max_tokens || pages + at.y + r.want - r.have > p.num_free)))
            atomicMin(&bad_request, b);
        tokens += all.x;
        pages += all.y;
    }
    __syncthreads();
    const int bad = bad_request;
    const bool fits = bad == 0x7fffffff;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.cu[0] = 0;
        p.taken[0] = fits ? (int)pages : 0;
        if (!fits) report(p.status, PTQ_ERR_INVALID_ARG, bad);
    }
    const long long used = fits ? tokens : 0;
    for (long long t = max(t0, used) + threadIdx.x; t < t1; t += kPlanThreads) { p.slots[t] = -1; p.positions[t] = -1; }
    if (!fits) {
        if (blockIdx.x == 0)
            for (int b = threadIdx.x; b < p.batch; b += kPlanThreads) { p.cu[b + 1] = 0; p.lens_out[b] = p.lens[b]; }
        return;
    }
    const bool again = p.batch > kPlanThreads;            // otherwise this thread's request is still at hand
    tokens = pages = 0;
    for (int first = 0; first < p.batch; first += kPlanThreads) {
        const int b = first + threadIdx.x;
        if (again) {
            r = plan_request(p, b);
            at = plan_scan(make_longlong2(r.n, r.want - r.have), warp_sums, all);
        }
        if (b < p.batch && blockIdx.x == 0) { p.cu[b + 1] = (int)(tokens + at.x + r.n); p.lens_out[b] = r.len + r.n; }
        const long long lo = max(t0, tokens), hi = min(t1, tokens + all.x);
        if (lo < hi) {                                    // the same for all threads
            at_token[threadIdx.x] = (int)(tokens + at.x);
            at_page[threadIdx.x] = (int)(pages + at.y);
            at_len[threadIdx.x] = r.len;
            at_have[threadIdx.x] = r.have;
            __syncthreads();
            for (long long t = lo + threadIdx.x; t < hi; t += kPlanThreads) {
                int i = 0;                                // the last request that begins at or before t: those behind it have tokens later
#pragma unroll
                for (int step = kPlanThreads / 2; step > 0; step >>= 1)
                    if (at_token[i + step] <= (int)t) i += step;
                const int pos = at_len[i] + (int)t - at_token[i], pi = pos >> p.page_shift, have = at_have[i];
                int32_t* row = p.table + (int64_t)(first + i) * p.ldt;
                const int page = pi >= have ? p.free_pages[at_page[i] + pi - have] : row[pi];
                if (pi >= have && (pos & (ps - 1)) == 0) row[pi] = page;
                const long long slot = ((long long)page << p.page_shift) + (pos & (ps - 1));
                const bool ok = page >= 0 && slot <= 0x7fffffffll;
                if (!ok) report(p.status, PTQ_ERR_INVALID_ARG, first + i, 1);
                p.slots[t] = ok ? (int)slot : -1;
                p.positions[t] = pos;
            }
            __syncthreads();
        }
        tokens += all.x;
        pages += all.y;
    }
}

// ------------------------------------------------------------------------------------------------------------
// Writing and reading
// ------------------------------------------------------------------------------------------------------------
// Step of a group with extremes lo <= 0 <= hi: (hi - lo) / 15 rounded up to 6 significant bits, as an fp16 pattern.
__device__ __forceinline__ uint32_t c4_step_bits(float lo, float hi) {
    const float r = fminf((hi - lo) / 15.0f, kC4MaxStep);
    const uint32_t h = __half_as_ushort(__float2half_ru(r));
    const uint32_t up = (h + 31u) & ~31u;
    return up < 32u ? 32u : up;                        // 32 is the pattern of 2^-19
}

struct C4Tokens {
    void* k;
    void* v;
    int64_t k_token, k_head, v_token, v_head;          // strides in elements; the head's values are contiguous
    const int32_t* slots;
    int tokens, vec;                                   // vec: every row begins on 16 bytes
    int32_t* status;
};

// Eight values a thread, four threads a group.  A step of decoding writes a few hundred rows and is bound by its launch (64 tokens, eight
// heads of 128: 4 us); many tokens are bound by instructions, the divisions first (16384 tokens 57 us, 1.5 TB/s, issue slots 80 % busy;
// reading them back 34 us, 2.5 TB/s, 74 %).
// A NaN is held as 0 and an infinity as the end of the grid (both recorded in status): the cache itself stays finite, so that a
// masked token can never reach a sum.
template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_append_kernel(Cache4 c, C4Tokens a) {
    chained_begin();
    constexpr int kRow = HD / 8;                                    // threads a row
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, row = u / kRow;
    const int sub = (int)(u - row * kRow);
    const int64_t th = row >> 1;
    const int token = (int)(th / c.kv_heads), head = (int)(th - (int64_t)token * c.kv_heads), side = (int)(row & 1);
    int slot = token < a.tokens ? a.slots[token] : -1;
    if (slot >= 0 && (slot >> c.page_shift) >= c.num_pages) {
        if (sub == 0) report(a.status, PTQ_ERR_INVALID_ARG, token);
        slot = -1;
    }
    float v[8];
    const T* src = side ? static_cast<const T*>(a.v) + token * a.v_token + head * a.v_head
                        : static_cast<const T*>(a.k) + token * a.k_token + head * a.k_head;
    load8<T>(src + sub * 8, slot >= 0 ? 8 : 0, a.vec, v);
    float lo = 0.f, hi = 0.f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        bad |= not_finite(v[i]);
        if (v[i] != v[i]) v[i] = 0.f;
        lo = fminf(lo, v[i]);
        hi = fmaxf(hi, v[i]);
    }
#pragma unroll
    for (int s = 1; s < 4; s <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, s));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, s));
    }
    if (slot < 0) return;
    if (bad) report(a.status, PTQ_ERR_NONFINITE, token);
    const uint32_t bits = c4_step_bits(lo, hi);
    const float step = __half2float(__ushort_as_half((unsigned short)bits));
    // true divisions: a tie between two codes is then a tie in any precision, and goes to the even one
    const float zero = fminf(fmaxf(rintf(-lo / step), 0.f), 15.f);
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float code = fminf(fmaxf(rintf(v[i] / step) + zero, 0.f), 15.f);
        codes |= (uint32_t)code << (4 * i);
    }
    const int in_page = slot & ((1 << c.page_shift) - 1), r = in_page & (kC4Tile - 1);
    uint8_t* tile = c4_tile<HD>(c, slot >> c.page_shift, head, in_page >> 4) + side * c4_side_bytes(HD);
    *reinterpret_cast<uint32_t*>(tile + r * (HD / 2) + sub * 4) = codes;
    if ((sub & 3) == 0)
        *reinterpret_cast<uint16_t*>(tile + kC4Tile * (HD / 2) + (r * (HD / kC4Group) + (sub >> 2)) * 2) = (uint16_t)(bits | (uint32_t)zero);
}

template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_read_kernel(Cache4 c, C4Tokens a) {
    chained_begin();
    constexpr int kRow = HD / 8;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x, row = u / kRow;
    const int sub = (int)(u - row * kRow);
    const int64_t th = row >> 1;
    const int token = (int)(th / c.kv_heads), head = (int)(th - (int64_t)token * c.kv_heads), side = (int)(row & 1);
    const int slot = token < a.tokens ? a.slots[token] : -1;
    if (slot < 0) return;
    if ((slot >> c.page_shift) >= c.num_pages) {
        if (sub == 0) report(a.status, PTQ_ERR_INVALID_ARG, token);
        return;
    }
    const int in_page = slot & ((1 << c.page_shift) - 1), r = in_page & (kC4Tile - 1);
    const uint8_t* tile = c4_tile<HD>(c, slot >> c.page_shift, head, in_page >> 4) + side * c4_side_bytes(HD);
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(tile + r * (HD / 2) + sub * 4);
    const uint32_t word = *reinterpret_cast<const uint16_t*>(tile + kC4Tile * (HD / 2) + (r * (HD / kC4Group) + (sub >> 2)) * 2);
    const float step = __half2float(__ushort_as_half((unsigned short)(word & 0xffe0u)));
    const int zero = (int)(word & 15u);
    alignas(16) T out[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = from_f32<T>(step * (float)((int)(codes >> (4 * i) & 15u) - zero));
    T* dst = side ? static_cast<T*>(a.v) + token * a.v_token + head * a.v_head : static_cast<T*>(a.k) + token * a.k_token + head * a.k_head;
    dst += sub * 8;
    if (a.vec) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(dst)[i] = reinterpret_cast<const uint4*>(out)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) dst[i] = out[i];
    }
}

// ------------------------------------------------------------------------------------------------------------
// Attention
// ------------------------------------------------------------------------------------------------------------
struct Attn4 {
    Cache4 cache;
    const void* q;
    void* out;
    float* lse;                                   // [total_q][q_heads] or NULL
    int64_t q_token, q_head, o_token, o_head;     // strides in elements
    const int32_t* table;
    int64_t ldt;
    int max_pages;
    const int32_t* lens;                          // [batch] tokens cached, the new ones among them
    const int32_t* cu;                            // [batch + 1] first row of each request
    int batch, total_q, q_heads, ratio;           // ratio = q_heads / kv_heads
    float scale_log2;                             // scale log2(e)
    int causal, window;
    int row_limit;                                // rows (new tokens x ratio) up to which a request is the business of the kernel for few
    int q_vec, o_vec;                             // every row of q / of out begins on 16 bytes
    uint2 by;                                     // {64, 4} (c4_unpack4)
    float* partial;
    int32_t* status;
};

// What beginning and ending a row tile costs a warp, in chunks.  With 0, 1, 2 (attention alone, us): 64 requests of up to 8192 tokens
// 131, 128, 128; two of up to 131072 82.1, 81.3, 80.7; 200 of up to 300 61, 65, 65.
constexpr int kFewTileCost = 1;

struct AttnRows { int row0, n, len; };                   // rows row0 .. row0 + n - 1, the last of len tokens
__device__ __forceinline__ AttnRows attn_rows(const Attn4& a, int b) {
    AttnRows r;
    const int c0 = a.cu[b], c1 = a.cu[b + 1], len = a.lens[b], most = a.max_pages << a.cache.page_shift;
    r.row0 = min(max(c0, 0), a.total_q);
    r.n = max(min(max(c1, 0), a.total_q) - r.row0, 0);
    r.len = min(max(len, 0), most);
    if (c0 != r.row0 || c1 != r.row0 + r.n || len != r.len) report(a.status, PTQ_ERR_INVALID_ARG, b);
    return r;
}

struct AttnRequest : AttnRows {
    int rows, tiles, chunk0, chunks;                     // tiles of kRows rows; kChunk-token chunks from chunk0 on
    long long units;
};
template <int kRows, int kChunk>
__device__ __forceinline__ AttnRequest attn_request(const Attn4& a, int b) {
    AttnRequest r;
    static_cast<AttnRows&>(r) = attn_rows(a, b);
    const long long rows = (long long)r.n * a.ratio;     // at most total_q q_heads < 2^31
    r.rows = rows > a.row_limit ? 0 : (int)rows;
    r.tiles = (r.rows + kRows - 1) / kRows;
    const int low = a.window > 0 ? (int)min(max((long long)r.len - r.n - a.window + 1, 0ll), (long long)r.len) : 0;
    r.chunk0 = low / kChunk;
    r.chunks = max((r.len + kChunk - 1) / kChunk - r.chunk0, 1);          // a request without keys still has rows to write
    r.units = (long long)a.cache.kv_heads * r.tiles * (r.chunks + kFewTileCost);
    return r;
}
// Keys [lo, hi) that row token i of the request sees.
__device__ __forceinline__ void attn_range(const Attn4& a, const AttnRows& r, int i, int& lo, int& hi) {
    const int pos = r.len - r.n + i;
    hi = a.causal ? min(max(pos + 1, 0), r.len) : r.len;
    lo = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
}

// Step and zero code of two 16-bit grid words to the factors that unpack their codes: with h = 1 + c / 16 (a nibble set into the
// mantissa of 1.0), s (c - z) = 16 s h - (16 + z) s.  16 s and (16 + z) s are exact in fp16 (6 and 11 significant bits), the
// difference has at most ten: the fused multiply-add rounds nothing.
struct C4Factors { __half2 step16, off; };
__device__ __forceinline__ C4Factors c4_factors(uint32_t words) {
    const uint32_t s = words & 0xffe0ffe0u, z = ((words & 0x000f000fu) << 6) | 0x4c004c00u;       // 16 + z
    const __half2 step = *reinterpret_cast<const __half2*>(&s), zero = *reinterpret_cast<const __half2*>(&z);
    C4Factors f;
    f.step16 = __hmul2(step, __float2half2_rn(16.f));
    f.off = __hneg2(__hmul2(step, zero));
    return f;
}
// Four values of either half.  The pipe of shifts and logic is the busiest one where codes are unpacked (66 % in the kernel for few rows,
// 60 % so; the times are the same within the noise), so shifts to the left are multiplications by `by` = {64, 4}, numbers that the
// compiler does not know and cannot make shifts of again.
// x: the lowest two nibbles of its halves are taken; y: those two that follow, at the same place.
__device__ __forceinline__ void c4_unpack4(uint32_t x, uint32_t y, const C4Factors& f, uint2 by, uint32_t (&o)[4]) {
    const uint32_t h[4] = {((x * by.x) & 0x03c003c0u) | 0x3c003c00u, ((x * by.y) & 0x03c003c0u) | 0x3c003c00u,
                           ((y * by.x) & 0x03c003c0u) | 0x3c003c00u, ((y * by.y) & 0x03c003c0u) | 0x3c003c00u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 v = __hfma2(*reinterpret_cast<const __half2*>(&h[i]), f.step16, f.off);
        o[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
}

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Power of two that brings a row of queries whose largest magnitude is `top` to [2^14, 2^15), so that bf16 queries become fp16
// ones: values down to 2^-31 of the row's largest stay as they are, smaller ones are off by at most 2^-39 of it.  1 for rows of zeros and
// for those that are not finite.
__device__ __forceinline__ int attn_q_shift(float top) {
    if (top == 0.f || not_finite(top)) return 0;
    return min(14 - ((int)(__float_as_uint(top) >> 23) - 127), 126);
}

// A negative scale changes the sign of q, a scale of 0 makes it 0, and the factor that the scores still need is positive.
__device__ __forceinline__ float attn_q_sign(float scale_log2) { return scale_log2 < 0.f ? -1.f : scale_log2 == 0.f ? 0.f : 1.f; }
__device__ __forceinline__ float attn_score_factor(float scale_log2, int shift) {
    // kept a finite normal number: times -infinity it has to stay -infinity, times 0 it has to stay 0
    return scale_log2 == 0.f ? 1.f : fminf(fmaxf(fabsf(scale_log2) * exp2_int(-shift), 1.17549435e-38f), 3.4e38f);
}

// Probabilities are kept times 2^15 in fp16: down to 2^-29 of the largest they keep all their bits, and nothing above 2^-39 of it
// is lost, so that many small ones still add up.
constexpr float kAttnPShift = 15.f;
// Natural logarithm of a row's sum of exponentials, kept as `sum` of 2^(x - ref + shift).
__device__ __forceinline__ float attn_lse(float ref, float sum, float shift) {
    return sum == 0.f ? -INFINITY : (ref + log2f(sum) - shift) * 0.693147180559945309f;
}

template <typename T> constexpr bool kIsHalf = false;
template <> constexpr bool kIsHalf<__half> = true;

// One CTA an SM: twelve warps with 168 registers each, or eight with up to 255 where a lane holds the output of sixteen rows.
__host__ __device__ constexpr int few_warps(int nt) { return nt == 1 ? 12 : 8; }
constexpr int kFewMaxCtas = 160, kFewChunk = 64, kFewTiles = kFewChunk / kC4Tile;
template <int HD, int NT> struct FewShape {
    static constexpr int warps = few_warps(NT), threads = 32 * warps;
    static constexpr int stages = HD == 128 ? 2 : 4;                  // 18432 bytes a warp either way
    static constexpr int chunk_bytes = kFewTiles * c4_tile_bytes(HD);
    static constexpr int smem_bytes = warps * stages * chunk_bytes + 128;
};
__host__ __device__ constexpr int few_partial_floats(int hd, int nt) { return 8 * nt * (hd + 2); }

// The units of all requests are dealt to the warps of the grid in equal shares, in the order (request, kv head, row tile, chunk): a
// long request and a batch of short ones fill the GPU alike.  A warp finds its share by adding up the requests' units, 256 at a time.
template <int W> struct FewScan { long long warp[W]; long long starts[32 * W]; };
template <int kRows, int W>
__device__ __forceinline__ long long few_total(const Attn4& a, FewScan<W>& s) {
    long long mine = 0;
    for (int b = threadIdx.x; b < a.batch; b += 32 * W) mine += attn_request<kRows, kFewChunk>(a, b).units;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
    if ((threadIdx.x & 31) == 0) s.warp[threadIdx.x >> 5] = mine;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) total += s.warp[w];
    __syncthreads();
    return total;
}
// The request that this warp's unit u belongs to and the units before it; all warps of the CTA, each with a u of its own (u >= total:
// none).
template <int kRows, int W>
__device__ __forceinline__ int few_find(const Attn4& a, long long u, FewScan<W>& s, long long& before) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long base = 0;
    int found = -1;
    for (int first = 0; first < a.batch; first += 32 * W) {
        const int b = first + threadIdx.x;
        const long long mine = b < a.batch ? attn_request<kRows, kFewChunk>(a, b).units : 0;
        long long x = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) s.warp[warp] = x;
        __syncthreads();
        long long all = 0, at = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w == warp) at = all;
            all += s.warp[w];
        }
        s.starts[threadIdx.x] = base + at + x - mine;
        __syncthreads();
        if (base <= u && u < base + all) {               // the last request that starts at or before u
            int count = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) count += __popc(__ballot_sync(0xffffffffu, s.starts[i * 32 + lane] <= u));
            found = first + count - 1;
            before = s.starts[count - 1];
        }
        base += all;
        __syncthreads();
    }
    return found;
}
__device__ __forceinline__ long long few_share(long long total, int workers) { return total > workers ? (total + workers - 1) / workers : 1; }

// A warp's part of a row tile: chunks [from, to), counted from the request's first.
struct FewPiece {
    AttnRequest r;
    int b, head, first_row, live_rows, from, to;
    int lo_any, hi_any, lo_all, hi_all;                  // keys that any, and that every row of the tile sees
    int c, c_end, last_tile;                             // its chunks that hold such keys, the end of its 16-token tiles
};
template <int kRows>
struct FewWalk {
    long long u, end, before;
    int b;
    __device__ __forceinline__ bool next(const Attn4& a, FewPiece& p) {
        while (u < end) {
            p.r = attn_request<kRows, kFewChunk>(a, b);
            if (u >= before + p.r.units) { before += p.r.units; ++b; continue; }
            const int length = p.r.chunks + kFewTileCost, seg = (int)((u - before) / length), x0 = (int)((u - before) - (long long)seg * length);
            const int x1 = (int)min((long long)length, x0 + (end - u));
            u += x1 - x0;
            p.from = max(x0 - kFewTileCost, 0);
            p.to = x1 - kFewTileCost;
            if (p.to <= p.from) continue;                // only what stands for the tile's beginning
            p.b = b;
            p.head = seg / p.r.tiles;
            p.first_row = (seg - p.head * p.r.tiles) * kRows;
            p.live_rows = min(kRows, p.r.rows - p.first_row);
            attn_range(a, p.r, p.first_row / a.ratio, p.lo_any, p.hi_all);
            attn_range(a, p.r, (p.first_row + p.live_rows - 1) / a.ratio, p.lo_all, p.hi_any);
            p.c = max(p.r.chunk0 + p.from, p.lo_any / kFewChunk);
            p.c_end = min(p.r.chunk0 + p.to, (p.hi_any + kFewChunk - 1) / kFewChunk);
            p.last_tile = (p.hi_any + kC4Tile - 1) / kC4Tile;
            return true;
        }
        return false;
    }
};

// Few rows (the new tokens of a request times the query heads of a kv head, up to 8 NT at a time): what counts is one read of the cache.
// Every warp works by itself, with two chunks of 64 tokens in flight (heads of 128; bulk copies, one for a tile); a row tile that
// lies in one warp's share is finished by it, others are joined afterwards.
// The cache is the 16-row operand of the tensor cores and the query rows their eight columns, so that a group of up to eight query
// heads costs half of what it would the other way round:  S^T = K q (16 tokens x 8 rows), O^T = V^T P^T (16 values x 8 rows).
// Codes go from shared memory to registers as they lie and become fp16 there: three instructions for two values.
// The order of a contraction is free, so the four lanes that share a token take 32 consecutive values each, and q is laid out alike.
// Two requests of 131072 and 81007 tokens, eight heads of 128: 67 us for 244 MB (3.6 TB/s); bound by the instructions that unpack: some
// 1600 for 64 tokens of a head, issued at 0.63 a clock, shifts and logic 60 % busy, the tensor cores 20 %.  (Sixteen warps with 32 tokens
// a turn 79 us; a CTA on one piece, its warps joined in shared memory, 81 us, and 140 against 95 for a ragged batch of 64.)
template <typename T, int HD, int NT>
__global__ void __launch_bounds__(32 * few_warps(NT), 1) attn4_few_kernel(Attn4 a) {
    using F = FewShape<HD, NT>;
    constexpr int kRows = 8 * NT, kWords = HD / 32, kSteps = HD / 16, kTiles = HD / 16, kLane = HD / 8;
    constexpr int kSide = c4_side_bytes(HD), kTileBytes = c4_tile_bytes(HD), kCodes = kC4Tile * HD / 2, kGrids = HD / kC4Group * 2;
    extern __shared__ unsigned char few_smem_raw[];
    __shared__ FewScan<F::warps> scan;
    __shared__ uint64_t bars[F::warps * F::stages];
    __shared__ int abort_word;
    unsigned char* ring = few_smem_raw + (128 - (smem_u32(few_smem_raw) & 127)) % 128;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n8 = lane >> 2, t = lane & 3;
    const unsigned char* ring_p = ring + warp * F::stages * F::chunk_bytes;
    const uint32_t ring_w = smem_u32(ring_p), bar_w = smem_u32(&bars[warp * F::stages]);
    if (lane < F::stages) mbar_init(bar_w + 8 * lane, 1);
    if (threadIdx.x == 0) abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    chained_begin();

    // workers side by side lie on different SMs: a small problem then uses as many of them as it has chunks
    const int worker = warp * gridDim.x + blockIdx.x, workers = F::warps * gridDim.x;
    const long long total = few_total<kRows>(a, scan), share = few_share(total, workers);
    FewWalk<kRows> walk;
    walk.u = share * worker;
    walk.end = min(walk.u + share, total);
    walk.before = 0;
    walk.b = few_find<kRows>(a, walk.u, scan, walk.before);

    unsigned asked = 0, done = 0;                        // chunks so far, over all pieces
    FewPiece p;
    int next = 0;
    auto ask = [&]() {                                   // the next chunk's tiles that hold keys; the whole warp
        const int stage = asked % F::stages, tile0 = next * kFewTiles, count = min(kFewTiles, p.last_tile - tile0);
        const uint32_t bar = bar_w + 8 * stage;
        if (lane == 0) mbar_arrive_expect_tx(bar, count * kTileBytes);
        __syncwarp();
        if (lane < count) {
            const int tl = tile0 + lane, per = a.cache.page_shift - 4;
            int page = a.table[(int64_t)p.b * a.ldt + (tl >> per)];
            if (page < 0 || page >= a.cache.num_pages) {
                // below the window there may be no page any more: some page's tokens, which are masked, stand in for them
                if (tl * kC4Tile + kC4Tile > p.lo_any) report(a.status, PTQ_ERR_INVALID_ARG, p.b, 2);
                page = 0;
            }
            bulk_load(ring_w + stage * F::chunk_bytes + lane * kTileBytes, c4_tile<HD>(a.cache, page, p.head, tl & ((1 << per) - 1)), kTileBytes, bar);
        }
        ++asked;
        ++next;
    };
    auto begin = [&]() {
        next = p.c;
#pragma unroll
        for (int s = 0; s < F::stages; ++s)
            if (next < p.c_end) ask();
    };
    bool more = walk.next(a, p), ok = true;
    if (more) begin();
    while (more && ok) {
        // the query rows, in the order in which the codes come
        uint32_t qf[NT][kSteps][2];
        float mult[NT][2];
        int lo[NT][2], hi[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = p.first_row + nt * 8 + n8;
            const bool live = row < p.r.rows;
            const int i = live ? row / a.ratio : 0;
            const T* q = static_cast<const T*>(a.q) + (int64_t)(p.r.row0 + i) * a.q_token + (int64_t)(p.head * a.ratio + (live ? row - i * a.ratio : 0)) * a.q_head;
            float v[kWords][8], top = 0.f;
            bool bad = false;
#pragma unroll
            for (int w = 0; w < kWords; ++w) load8<T>(q + (t * kWords + w) * 8, live ? 8 : 0, a.q_vec, v[w]);
#pragma unroll
            for (int w = 0; w < kWords; ++w)
#pragma unroll
                for (int e = 0; e < 8; ++e) { top = fmaxf(top, fabsf(v[w][e])); bad |= not_finite(v[w][e]); }
            if (bad) top = __uint_as_float(0x7f800000u);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int shift = kIsHalf<T> ? 0 : attn_q_shift(top);
            const float f = attn_q_sign(a.scale_log2) * exp2_int(shift);
#pragma unroll
            for (int w = 0; w < kWords; ++w)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    qf[nt][2 * w + h][0] = pack_half2(v[w][2 * h] * f, v[w][2 * h + 4] * f);
                    qf[nt][2 * w + h][1] = pack_half2(v[w][2 * h + 1] * f, v[w][2 * h + 5] * f);
                }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int rr = p.first_row + nt * 8 + 2 * t + h;
                mult[nt][h] = attn_score_factor(a.scale_log2, __shfl_sync(0xffffffffu, shift, (2 * t + h) * 4));
                lo[nt][h] = hi[nt][h] = 0;
                if (rr < p.r.rows) attn_range(a, p.r, rr / a.ratio, lo[nt][h], hi[nt][h]);
            }
        }

        float m[NT][2], l[NT][2], o[NT][kTiles][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int h = 0; h < 2; ++h) { m[nt][h] = -INFINITY; l[nt][h] = 0.f; }
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][j][e] = 0.f;
        }
        // one chunk; `masked`: some row does not see all of it
        auto chunk = [&](const unsigned char* data, int j0, auto masked) {
            constexpr bool kMasked = decltype(masked)::value;
            float x[NT][kFewTiles][4];
#pragma unroll
            for (int tl = 0; tl < kFewTiles; ++tl) {
                const unsigned char* side = data + tl * kTileBytes;
                alignas(16) uint32_t kw[2][kWords];
                C4Factors f[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int token = n8 + 8 * h;
                    if constexpr (HD == 128) *reinterpret_cast<uint4*>(kw[h]) = *reinterpret_cast<const uint4*>(side + token * (HD / 2) + t * 16);
                    else *reinterpret_cast<uint2*>(kw[h]) = *reinterpret_cast<const uint2*>(side + token * (HD / 2) + t * 8);
                    const uint32_t g = *reinterpret_cast<const uint16_t*>(side + kCodes + token * kGrids + t * 8 * kWords / kC4Group * 2);
                    f[h] = c4_factors(__byte_perm(g, g, 0x1010));
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[nt][tl][e] = 0.f;
#pragma unroll
                for (int w = 0; w < kWords; ++w) {
                    uint32_t k0[4], k1[4];
                    c4_unpack4(kw[0][w], kw[0][w] >> 8, f[0], a.by, k0);
                    c4_unpack4(kw[1][w], kw[1][w] >> 8, f[1], a.by, k1);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            mma_f16(x[nt][tl], k0[2 * h], k1[2 * h], k0[2 * h + 1], k1[2 * h + 1], qf[nt][2 * w + h][0], qf[nt][2 * w + h][1]);
                }
            }
            // softmax: the reference m (a score, before its factor) is raised only when some score lies above it
            float top[NT][2];
            bool above = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    top[nt][h] = m[nt][h];
#pragma unroll
                    for (int tl = 0; tl < kFewTiles; ++tl)
#pragma unroll
                        for (int e = h; e < 4; e += 2) {
                            if (kMasked) {
                                const int j = j0 + tl * kC4Tile + n8 + 8 * (e >> 1);
                                if (j < lo[nt][h] || j >= hi[nt][h]) x[nt][tl][e] = -INFINITY;
                            }
                            top[nt][h] = fmaxf(top[nt][h], x[nt][tl][e]);
                        }
                    above |= top[nt][h] > m[nt][h];
                }
            if (__any_sync(0xffffffffu, above)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top[nt][h] = fmaxf(top[nt][h], __shfl_xor_sync(0xffffffffu, top[nt][h], d));
                        const float f = m[nt][h] == top[nt][h] ? 1.f : exp2_approx((m[nt][h] - top[nt][h]) * mult[nt][h]);    // 0 from -infinity
                        m[nt][h] = top[nt][h];
                        l[nt][h] *= f;
#pragma unroll
                        for (int j = 0; j < kTiles; ++j) { o[nt][j][h] *= f; o[nt][j][h + 2] *= f; }
                    }
            }
            uint32_t pf[NT][kFewTiles][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                // The difference comes before the factor: a product of the reference is off by up to half a step of its own, more
                // than fp16 has room for once scores pass 2^23.  Two at a time this costs what one fused operation each does.
                const float2 factor = make_float2(mult[nt][0], mult[nt][1]), shift = make_float2(kAttnPShift, kAttnPShift);
                const float2 minus_ref = make_float2(m[nt][0] == -INFINITY ? 0.f : -m[nt][0], m[nt][1] == -INFINITY ? 0.f : -m[nt][1]);
                float2 part = make_float2(0.f, 0.f);
#pragma unroll
                for (int tl = 0; tl < kFewTiles; ++tl) {
                    float pr[4];
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const float2 y = fma2(add2(make_float2(x[nt][tl][e], x[nt][tl][e + 1]), minus_ref), factor, shift);
                        pr[e] = exp2_approx(y.x);
                        pr[e + 1] = exp2_approx(y.y);
                        part = add2(part, make_float2(pr[e], pr[e + 1]));
                    }
                    pf[nt][tl][0] = transpose8(pack_half2(pr[0], pr[1]));
                    pf[nt][tl][1] = transpose8(pack_half2(pr[2], pr[3]));
                }
                l[nt][0] += part.x;
                l[nt][1] += part.y;
            }
#pragma unroll
            for (int tl = 0; tl < kFewTiles; ++tl) {
                const unsigned char* side = data + tl * kTileBytes + kSide;
                constexpr int kV = HD / 64;                       // words a lane: 16 or 8 values of a token
                alignas(8) uint32_t vw[4][kV];
                uint32_t g[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int token = 2 * t + (e & 1) + 8 * (e >> 1);
                    if constexpr (HD == 128) *reinterpret_cast<uint2*>(vw[e]) = *reinterpret_cast<const uint2*>(side + token * (HD / 2) + n8 * 8);
                    else vw[e][0] = *reinterpret_cast<const uint32_t*>(side + token * (HD / 2) + n8 * 4);
                    g[e] = *reinterpret_cast<const uint16_t*>(side + kCodes + token * kGrids + n8 * 8 * kV / kC4Group * 2);
                    if (kMasked) {                                // what nobody sees may hold anything: 0 times it has to be 0
                        const int j = j0 + tl * kC4Tile + token;
                        if (j < p.lo_any || j >= p.hi_any) g[e] = 0u;
                    }
                }
                const C4Factors f0 = c4_factors(__byte_perm(g[0], g[1], 0x5410)), f1 = c4_factors(__byte_perm(g[2], g[3], 0x5410));
#pragma unroll
                for (int w = 0; w < kV; ++w)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t v0[4], v1[4];
                        c4_unpack4(__byte_perm(vw[0][w], vw[1][w], h ? 0x7632 : 0x5410), __byte_perm(vw[0][w], vw[1][w], h ? 0x0703 : 0x0501), f0, a.by, v0);
                        c4_unpack4(__byte_perm(vw[2][w], vw[3][w], h ? 0x7632 : 0x5410), __byte_perm(vw[2][w], vw[3][w], h ? 0x0703 : 0x0501), f1, a.by, v1);
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                mma_f16(o[nt][4 * w + 2 * h + e], v0[2 * e], v0[2 * e + 1], v1[2 * e], v1[2 * e + 1], pf[nt][tl][0], pf[nt][tl][1]);
                    }
            }
        };
        for (int c = p.c; c < p.c_end; ++c) {
            const int stage = done % F::stages, j0 = c * kFewChunk;
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(bar_w + 8 * stage, (done / F::stages) & 1, &abort_word));
            if (!ok) break;
            ++done;
            if (j0 >= p.lo_all && j0 + kFewChunk <= p.hi_all) chunk(ring_p + stage * F::chunk_bytes, j0, std::false_type());
            else chunk(ring_p + stage * F::chunk_bytes, j0, std::true_type());
            __syncwarp();                                         // the stage has been read
            if (next < p.c_end) ask();
        }
        if (!ok) {                                                // copies in flight land before the CTA is left
            for (; done < asked; ++done) drain_copy(bar_w + 8 * (done % F::stages), (done / F::stages) & 1);
            if (lane == 0) report(a.status, PTQ_ERR_TIMEOUT, blockIdx.x, 3);
            break;
        }
        // the next piece's first chunks are under way while this one's results are written
        const FewPiece old = p;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) m[nt][h] = m[nt][h] == -INFINITY ? -INFINITY : m[nt][h] * mult[nt][h];
        more = walk.next(a, p);
        if (more) begin();
        const bool complete = old.from == 0 && old.to == old.r.chunks;
        float* slot = a.partial + (int64_t)(2 * worker + (old.from == 0 ? 1 : 0)) * few_partial_floats(HD, NT);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[nt][h] += __shfl_xor_sync(0xffffffffu, l[nt][h], d);
                const int in = nt * 8 + 2 * t + h;
                if (in >= old.live_rows) continue;
                float v[kLane];
                if (complete) {
                    const float inv = l[nt][h] == 0.f ? 0.f : 1.f / l[nt][h];
#pragma unroll
                    for (int j = 0; j < kTiles; ++j) { v[2 * j] = o[nt][j][h] * inv; v[2 * j + 1] = o[nt][j][h + 2] * inv; }
                    const int rr = old.first_row + in, i = rr / a.ratio, qh = old.head * a.ratio + rr - i * a.ratio;
                    store_row<T, kLane>(static_cast<T*>(a.out) + (int64_t)(old.r.row0 + i) * a.o_token + (int64_t)qh * a.o_head + n8 * kLane, v, a.o_vec);
                    if (n8 == 0 && a.lse)
                        a.lse[(int64_t)(old.r.row0 + i) * a.q_heads + qh] = attn_lse(m[nt][h] == -INFINITY ? 0.f : m[nt][h], l[nt][h], kAttnPShift);
                } else {
#pragma unroll
                    for (int j = 0; j < kTiles; ++j) { v[2 * j] = o[nt][j][h]; v[2 * j + 1] = o[nt][j][h + 2]; }
                    store_row<float, kLane>(slot + in * HD + n8 * kLane, v, true);
                    if (n8 == 0) { slot[kRows * HD + in] = m[nt][h]; slot[kRows * (HD + 1) + in] = l[nt][h]; }
                }
            }
    }
}

// Joins the partial results of row tiles that several warps shared.  Warp w of CTA c looks at the border behind worker
// 8 c + w: if it is the first one inside a tile, the CTA adds up that tile's pieces, in their order: a warp a row, or, where
// the pieces are many, all warps a row together, each an eighth of the pieces.
constexpr int kJoinTogether = 16, kJoinWarps = 8, kJoinThreads = 32 * kJoinWarps;
template <typename T, int HD, int NT>
__global__ void __launch_bounds__(kJoinThreads) attn4_join_kernel(Attn4 a, int ctas) {
    constexpr int kRows = 8 * NT, kLane = HD / 32;
    __shared__ FewScan<kJoinWarps> scan;
    struct Job { int b, head, tile, w0, w1; };
    __shared__ Job jobs[kJoinWarps];
    __shared__ float part_top[kJoinWarps], part_sum[kJoinWarps], part_v[kJoinWarps][HD];
    chained_begin();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, workers = ctas * few_warps(NT), border = blockIdx.x * kJoinWarps + warp;
    const long long total = few_total<kRows>(a, scan), share = few_share(total, workers), u = share * (border + 1);
    if (share * (blockIdx.x * kJoinWarps + 1) >= total) return;
    long long before = 0;
    const int b = few_find<kRows>(a, u, scan, before);
    Job mine{-1, 0, 0, 0, 0};
    if (b >= 0) {
        const AttnRequest r = attn_request<kRows, kFewChunk>(a, b);
        const int length = r.chunks + kFewTileCost, seg = (int)((u - before) / length);
        const long long s0 = before + (long long)seg * length + kFewTileCost;          // its first chunk
        const long long w0 = s0 / share, w1 = (s0 + r.chunks - 1) / share;
        if (u > s0 && w0 == border) mine = Job{b, seg / r.tiles, seg % r.tiles, (int)w0, (int)w1};
    }
    if (lane == 0) jobs[warp] = mine;
    __syncthreads();
    auto weight = [&](int w, int w0, int row) -> const float* {
        return a.partial + (int64_t)(2 * w + (w == w0)) * few_partial_floats(HD, NT) + kRows * HD + row;
    };
    auto finish = [&](const AttnRequest& r, const Job& j, int row, float ref, float sum, const float (&v)[kLane]) {
        const int rr = j.tile * kRows + row, i0 = rr / a.ratio, qh = j.head * a.ratio + rr - i0 * a.ratio;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        T* out = static_cast<T*>(a.out) + (int64_t)(r.row0 + i0) * a.o_token + (int64_t)qh * a.o_head + lane * kLane;
#pragma unroll
        for (int i = 0; i < kLane; ++i) out[i] = from_f32<T>(v[i] * inv);
        if (lane == 0 && a.lse) a.lse[(int64_t)(r.row0 + i0) * a.q_heads + qh] = attn_lse(ref, sum, kAttnPShift);
    };
    for (int k = 0; k < kJoinWarps; ++k) {
        const Job j = jobs[k];
        if (j.b < 0) continue;
        const AttnRequest r = attn_request<kRows, kFewChunk>(a, j.b);
        const int live_rows = min(kRows, r.rows - j.tile * kRows);
        const bool together = j.w1 - j.w0 >= kJoinTogether;
        for (int row = together ? 0 : warp; row < live_rows; row += together ? 1 : kJoinWarps) {
            const int step = together ? kJoinWarps : 1, w_first = j.w0 + (together ? warp : 0);
            float top = -INFINITY, sum = 0.f, v[kLane];
#pragma unroll
            for (int i = 0; i < kLane; ++i) v[i] = 0.f;
            for (int w = w_first + lane * step; w <= j.w1; w += 32 * step) top = fmaxf(top, *weight(w, j.w0, row));
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll 4
            for (int w = w_first; w <= j.w1; w += step) {
                const float* stat = weight(w, j.w0, row);
                const float f = exp2_approx(stat[0] - ref);
                sum += f * stat[kRows];
#pragma unroll
                for (int i = 0; i < kLane; ++i) v[i] += f * stat[row * HD - kRows * HD - row + lane * kLane + i];
            }
            if (!together) {
                finish(r, j, row, ref, sum, v);
                continue;
            }
            if (lane == 0) { part_top[warp] = top; part_sum[warp] = sum; }
#pragma unroll
            for (int i = 0; i < kLane; ++i) part_v[warp][lane * kLane + i] = v[i];
            __syncthreads();
            if (warp == 0) {
                float all_top = -INFINITY, all = 0.f, w[kLane];
                for (int q = 0; q < kJoinWarps; ++q) all_top = fmaxf(all_top, part_top[q]);
                const float all_ref = all_top == -INFINITY ? 0.f : all_top;
#pragma unroll
                for (int i = 0; i < kLane; ++i) w[i] = 0.f;
                for (int q = 0; q < kJoinWarps; ++q) {
                    const float f = exp2_approx(part_top[q] - all_ref);
                    all += f * part_sum[q];
#pragma unroll
                    for (int i = 0; i < kLane; ++i) w[i] += f * part_v[q][lane * kLane + i];
                }
                finish(r, j, row, all_ref, all, w);
            }
            __syncthreads();
        }
    }
}

}  // namespace ptq
