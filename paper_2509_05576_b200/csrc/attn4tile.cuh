// Attention of many rows (prompts) over the 4-bit cache, on tcgen05.
//
// A CTA takes 256 query rows of one request and kv head (tokens x query heads of the group) as two tiles of 128, and 128 keys at a
// time: one unpacking of the cache serves both.  Four warps unpack (the codes come from L2 straight into registers, one chunk ahead) and
// write K [128 keys][dim] and V^T [dim][128 keys] as fp16, K-major, SWIZZLE_128B, into one of two stages; one thread issues
// S = Q K^T and O += P V; four warps for each tile, a row a thread, turn S into P.  While one tile's softmax runs, the tensor cores
// work on the other tile.  TMEM (all 512 columns): S0, S1 (128 each), O0, O1.  P is fp16 and lies where its S was, as the operand
// of the second product.
//
// Per chunk the tensor cores need 2 x 1024 clocks (heads of 128), the exponentials 2 x 1024 (16 a clock); a chunk takes some 4700.
// 1024 and 633 tokens behind 7168 and 4430, 32 heads on 8: 195 us, 0.9 PFLOP/s.  No part bounds it alone: without the
// exponentials, without unpacking or with an eighth of the products it is 13, 10 or 15 us faster, without all of them 76; what is left is
// the chain scores - softmax - products of each tile, and four unpacking warps whose loads and shared-memory stores take 4300 clocks a
// chunk.  Tried, and slower or no faster: seven unpacking warps with items unrolled (358 us: the four roles then wait for
// instructions) or rolled (253), codes through shared memory by bulk copies (213), keys and values in stages of their own (203),
// scores in halves of 64 keys so that a tile's next scores are formed during its softmax (238), one pass over the scores with the
// probabilities held in registers (267).
// The reference of a row's exponentials is only moved when a score lies more than 2^7 above it (P then still fits fp16), so that O is
// hardly ever rescaled.
//
// 128 registers a thread at launch, dealt out by role; the compiler spills 32 bytes a thread (heads of 128).
//
// The units (128 keys of one tile) are dealt to the CTAs in equal shares, as those of the kernel for few rows; what a row tile sees of
// the keys differs from tile to tile, so a first small kernel lists the tiles with the units before each.
#pragma once
#include "cache4.cuh"

namespace ptq {

constexpr int kTileRows = 256, kTileKeys = 128, kTileThreads = 512, kTileMaxCtas = 160, kScheduleThreads = 1024;
// What beginning and ending a tile costs a CTA, in chunks.  With 0, 1, 2 (attention alone, us): six prompts of 1500 tokens, heads of 64
// 143, 106, 94; two of 1024 tokens behind up to 7168, heads of 128 264, 265, 256.
constexpr int kTileCost = 1;
constexpr float kTilePShift = 8.f, kTileSlack = 7.f;     // P = 2^(x - ref + 8) <= 2^15

template <int HD> struct TileShape {
    static constexpr int q_bytes = 2 * 128 * HD * 2;                          // both tiles
    static constexpr int k_bytes = kTileKeys * HD * 2, stage_bytes = 2 * k_bytes;
    static constexpr int smem_bytes = 1024 + q_bytes + 2 * stage_bytes + 256;
};
__host__ __device__ constexpr int64_t tile_partial_floats(int hd) { return (int64_t)kTileRows * (hd + 2); }

struct TileList {
    long long* before;        // [count + 1] units (of one kv head) before each tile; before[most + 1] holds the count
    int2* tile;               // [count] request, row tile
    int most;                 // room
};

struct TileRange { int lo_any, hi_any, lo_all, hi_all, chunk0, chunks; };
// Keys that any and that every row of a tile sees, and its 128-key chunks.
__device__ __forceinline__ TileRange tile_range(const Attn4& a, const AttnRows& r, int tile) {
    TileRange t;
    const int first = tile * kTileRows, last = min(first + kTileRows, r.n * a.ratio) - 1;
    attn_range(a, r, first / a.ratio, t.lo_any, t.hi_all);
    attn_range(a, r, last / a.ratio, t.lo_all, t.hi_any);
    t.chunk0 = min(t.lo_any, t.hi_any) / kTileKeys;
    t.chunks = max((t.hi_any + kTileKeys - 1) / kTileKeys - t.chunk0, 1);     // a tile without keys still has rows to write
    return t;
}

__global__ void __launch_bounds__(kScheduleThreads) attn4_schedule_kernel(Attn4 a, TileList list) {
    chained_begin();
    __shared__ longlong2 warp_sums[32];
    __shared__ int first_tile[kScheduleThreads + 1];
    long long units = 0;
    int count = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kScheduleThreads) {
        // tiles of these requests, then all their tiles side by side
        int mine = 0;
        if (b0 + (int)threadIdx.x < a.batch) {
            const long long rows = (long long)attn_rows(a, b0 + threadIdx.x).n * a.ratio;
            mine = rows > a.row_limit ? (int)((rows + kTileRows - 1) / kTileRows) : 0;
        }
        longlong2 all;
        first_tile[threadIdx.x] = (int)plan_scan(make_longlong2(mine, 0), warp_sums, all).x;
        const int tiles = (int)all.x;
        if (threadIdx.x == 0) first_tile[kScheduleThreads] = tiles;
        __syncthreads();
        for (int f0 = 0; f0 < tiles; f0 += kScheduleThreads) {
            const int f = f0 + threadIdx.x;
            int b = 0, tile = 0, chunks = 0;
            if (f < tiles) {
                int lo = 0, hi = kScheduleThreads;                            // first_tile[lo] <= f < first_tile[hi]
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (first_tile[mid] <= f) lo = mid; else hi = mid;
                }
                b = b0 + lo;
                tile = f - first_tile[lo];
                chunks = tile_range(a, attn_rows(a, b), tile).chunks + kTileCost;
            }
            const longlong2 at = plan_scan(make_longlong2(chunks, 0), warp_sums, all);
            if (f < tiles && count + f < list.most) {
                list.before[count + f] = units + at.x;
                list.tile[count + f] = make_int2(b, tile);
            }
            units += all.x;
        }
        count += tiles;
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        count = min(count, list.most);
        list.before[count] = units;
        list.before[list.most + 1] = count;
    }
}

// A CTA's way through its share of the units.
struct TilePiece {
    int b, tile, head, from, to;         // chunks [from, to) of the tile, counted from its first
    AttnRows r;
    TileRange range;
};
struct TileWalk {
    long long u, end, share;
    int f;
    __device__ __forceinline__ bool next(const Attn4& a, const TileList& list, TilePiece& p) {
        const long long heads = a.cache.kv_heads;
        while (u < end) {
            while (u >= heads * list.before[f + 1]) ++f;
            const long long base = list.before[f], length = list.before[f + 1] - base, rel = u - heads * base;
            p.head = (int)(rel / length);
            const int x0 = (int)(rel - p.head * length), x1 = (int)min(length, x0 + (end - u));
            u += x1 - x0;
            p.from = max(x0 - kTileCost, 0);
            p.to = x1 - kTileCost;
            if (p.to <= p.from) continue;                // only what stands for the tile's beginning
            const int2 t = list.tile[f];
            p.b = t.x;
            p.tile = t.y;
            p.r = attn_rows(a, p.b);
            p.range = tile_range(a, p.r, p.tile);
            return true;
        }
        return false;
    }
};
__device__ __forceinline__ long long tile_share(long long total, int ctas) { return (total + ctas - 1) / ctas; }
// The tile that unit u (of all heads) lies in: the threads of the CTA look side by side.
__device__ __forceinline__ void tile_find(const Attn4& a, const TileList& list, int count, long long u, int* found) {
    for (int f = threadIdx.x; f < count; f += blockDim.x)
        if (a.cache.kv_heads * list.before[f] <= u && u < a.cache.kv_heads * list.before[f + 1]) *found = f;
    __syncthreads();
}

__host__ __device__ constexpr uint32_t f16_idesc(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24); }
__device__ __forceinline__ void tc_mma_f16(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
                 "mov.b64 da, {%1, %3};\n\t"
                 "mov.b64 db, {%2, %3};\n\t"
                 "setp.ne.b32 p, %5, 0;\n\t"
                 "elect.sync _|e, 0xffffffff;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, {%6, %6, %6, %6}, p;\n\t}\n"
                 ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(kF8DescHi), "r"(idesc), "r"(accumulate), "r"(0u)
                 : "memory");
}
// The row operand in TMEM, two fp16 a column.
__device__ __forceinline__ void tc_mma_f16_tmem(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 db;\n\t"
                 "mov.b64 db, {%2, %3};\n\t"
                 "setp.ne.b32 p, %5, 0;\n\t"
                 "elect.sync _|e, 0xffffffff;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, {%6, %6, %6, %6}, p;\n\t}\n"
                 ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(kF8DescHi), "r"(idesc), "r"(accumulate), "r"(0u)
                 : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Loads that stay where they are written: a chunk's are issued before the wait for room, a whole chunk ahead of their use.
__device__ __forceinline__ uint4 ld_global16(const uint8_t* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ld_global4(const uint8_t* p) {
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ld_global2(const uint8_t* p) {
    uint16_t v;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
    return v;
}

// Place of 16-byte piece c of row `row` in a K-major operand of `rows` rows, 64 values (128 bytes) a slab, SWIZZLE_128B.
__device__ __forceinline__ uint32_t tile_at(int rows, int row, int c) {
    return (uint32_t)((c >> 3) * rows * 128 + row * 128 + (((c & 7) ^ (row & 7)) << 4));
}

// Keys [lo, hi) of a row among the 32 from `at` on, a bit each.
__device__ __forceinline__ uint32_t tile_seen(int lo, int hi, int at) {
    const int a = min(max(lo - at, 0), 32), b = min(max(hi - at, 0), 32);
    return (b == 32 ? 0xffffffffu : (1u << b) - 1u) & ~(a == 32 ? 0xffffffffu : (1u << a) - 1u);
}
// A row's largest score of the chunk, and its probabilities, written where the scores were (two fp16 a column), with their sum.
// kWhole: the row sees all 128 keys; otherwise keys [lo, hi).  The scores are read twice rather than kept in 128 registers.
template <bool kWhole>
__device__ __forceinline__ float tile_max(uint32_t s_tmem, int lo, int hi) {
    float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    uint32_t r[2][32];                                   // 32 scores are read while the 32 before them are looked at
    tc_ld32(s_tmem, r[0]);
#pragma unroll
    for (int ch = 0; ch < 4; ++ch) {
        const uint32_t seen = kWhole ? 0u : tile_seen(lo, hi, ch * 32);
        tc_wait_ld();
        if (ch < 3) tc_ld32(s_tmem + (ch + 1) * 32, r[(ch + 1) & 1]);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            const float v = kWhole || (seen >> e & 1u) ? __uint_as_float(r[ch & 1][e]) : -INFINITY;
            top[e & 3] = fmaxf(top[e & 3], v);
        }
    }
    return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}
template <bool kWhole>
__device__ __forceinline__ float tile_probs(uint32_t s_tmem, float mult, float off, int lo, int hi) {
    float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    uint32_t r[2][32];
    tc_ld32(s_tmem, r[0]);
#pragma unroll
    for (int ch = 0; ch < 4; ++ch) {
        uint32_t w[16];
        const uint32_t seen = kWhole ? 0u : tile_seen(lo, hi, ch * 32);
        tc_wait_ld();
        if (ch < 3) tc_ld32(s_tmem + (ch + 1) * 32, r[(ch + 1) & 1]);
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float2 x = fma2(make_float2(__uint_as_float(r[ch & 1][e]), __uint_as_float(r[ch & 1][e + 1])), make_float2(mult, mult), make_float2(off, off));
            float v0 = exp2_approx(x.x), v1 = exp2_approx(x.y);
            if (!kWhole) {
                v0 = seen >> e & 1u ? v0 : 0.f;
                v1 = seen >> (e + 1) & 1u ? v1 : 0.f;
            }
            part[(e >> 1) & 1] = add2(part[(e >> 1) & 1], make_float2(v0, v1));
            w[e >> 1] = pack_half2(v0, v1);
        }
        tc_st16(s_tmem + ch * 16, w);
    }
    return (part[0].x + part[0].y) + (part[1].x + part[1].y);
}

// An exponent is (score mult + off), off = 8 - reference mult: one operation for two of them, but off is rounded, by up to half a step of
// its own.  Up to kTileFar that is a quarter at most, and 2^15.25 an fp16 number still; beyond, the reference is taken from the score
// before the factor is applied.  Rare, so short rather than fast: a third copy of the loop above, never entered, made everything slower
// (1024 and 633 tokens behind 7168 and 4430: 229 -> 240 us).
constexpr float kTileFar = 4194304.f;
__device__ __noinline__ float tile_probs_far(uint32_t s_tmem, float mult, float ref, int lo, int hi) {
    float sum = 0.f;
#pragma unroll 1
    for (int ch = 0; ch < 8; ++ch) {
        uint32_t r[16], w[8];
        tc_ld16(s_tmem + ch * 16, r);
        tc_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const int j = ch * 16 + e;
            const float v0 = j >= lo && j < hi ? exp2_approx(fmaf(__uint_as_float(r[e]) - ref, mult, kTilePShift)) : 0.f;
            const float v1 = j + 1 >= lo && j + 1 < hi ? exp2_approx(fmaf(__uint_as_float(r[e + 1]) - ref, mult, kTilePShift)) : 0.f;
            sum += v0 + v1;
            w[e >> 1] = pack_half2(v0, v1);
        }
        tc_st8(s_tmem + ch * 8, w);
    }
    return sum;
}

template <typename T, int HD>
__global__ void __launch_bounds__(kTileThreads, 1) attn4_tile_kernel(Attn4 a, TileList list) {
    using S = TileShape<HD>;
    constexpr int kSide = c4_side_bytes(HD), kCodes = kC4Tile * HD / 2, kGrids = HD / kC4Group * 2;
    extern __shared__ unsigned char tile_smem_raw[];
    __shared__ int found, abort_word;
    const uint32_t raw = smem_u32(tile_smem_raw), base = (raw + 1023u) & ~1023u;
    unsigned char* base_ptr = tile_smem_raw + (base - raw);
    unsigned char* tail = base_ptr + S::q_bytes + 2 * S::stage_bytes;
    const uint32_t bar0 = smem_u32(tail);
    auto q_full = [&](int t) { return bar0 + 8u * t; };
    auto kv_full = [&](int s) { return bar0 + 8u * (2 + s); };
    auto kv_empty = [&](int s) { return bar0 + 8u * (4 + s); };
    auto s_full = [&](int t) { return bar0 + 8u * (6 + t); };
    auto p_full = [&](int t) { return bar0 + 8u * (8 + t); };
    auto o_full = [&](int t) { return bar0 + 8u * (10 + t); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 8 * 12);
    volatile int* abort_flag = &abort_word;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full(i), 128);
            mbar_init(kv_full(i), 128);
            mbar_init(kv_empty(i), 1);
            mbar_init(s_full(i), 1);
            mbar_init(p_full(i), 128);
            mbar_init(o_full(i), 1);
        }
        abort_word = 0;
        found = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 12) tc_alloc(smem_u32(tmem_slot), 512u);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
    chained_wait();

    const int count = (int)list.before[list.most + 1];
    const long long total = a.cache.kv_heads * list.before[count];
    TileWalk walk;
    walk.share = tile_share(total, gridDim.x);
    walk.u = walk.share * blockIdx.x;
    walk.end = min(walk.u + walk.share, total);
    if (walk.u < walk.end) tile_find(a, list, count, walk.u, &found);      // the same for all threads
    walk.f = found;
    TilePiece p;

    if (warp < 8) {
        // ------------------------------------------------------------ softmax: a row a thread
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
        const int t = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_tmem = tmem + lanes + t * 128, o_tmem = tmem + lanes + 256 + t * 128;
        unsigned char* q_smem = base_ptr + t * (S::q_bytes / 2);
        uint32_t s_phase = 0, o_phase = 0;
        bool ok = true;
        while (ok && walk.next(a, list, p)) {
            const int rows = p.r.n * a.ratio, first = p.tile * kTileRows, rr = first + t * 128 + row;
            if (t == 1 && rows - first <= 128) continue;                      // the second tile is empty
            const bool live = rr < rows;
            const int i = live ? rr / a.ratio : 0, qh = p.head * a.ratio + (live ? rr - i * a.ratio : 0);
            // the row's queries, as fp16 in the order in which the codes come
            float mult = 0.f;
            {
                const T* q = static_cast<const T*>(a.q) + (int64_t)(p.r.row0 + i) * a.q_token + (int64_t)qh * a.q_head;
                uint4 raw[HD / 8];                       // the whole row at once: one trip to memory
                if (live && a.q_vec) {
#pragma unroll
                    for (int c = 0; c < HD / 8; ++c) raw[c] = reinterpret_cast<const uint4*>(q)[c];
                } else {
#pragma unroll
                    for (int c = 0; c < HD / 8; ++c) {
                        T* e = reinterpret_cast<T*>(&raw[c]);
#pragma unroll
                        for (int k = 0; k < 8; ++k) e[k] = live ? q[8 * c + k] : from_f32<T>(0.f);
                    }
                }
                float top = 0.f;
                bool bad = false;
#pragma unroll
                for (int c = 0; c < HD / 8; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float v = to_f32<T>(reinterpret_cast<const T*>(&raw[c])[e]);
                        top = fmaxf(top, fabsf(v));
                        bad |= not_finite(v);
                    }
                const int shift = kIsHalf<T> || bad ? 0 : attn_q_shift(top);
                const float f = attn_q_sign(a.scale_log2) * exp2_int(shift);
                mult = attn_score_factor(a.scale_log2, shift);
#pragma unroll
                for (int c = 0; c < HD / 8; ++c) {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = to_f32<T>(reinterpret_cast<const T*>(&raw[c])[e]) * f;
                    *reinterpret_cast<uint4*>(q_smem + tile_at(128, row, c)) =
                        make_uint4(pack_half2(v[0], v[4]), pack_half2(v[1], v[5]), pack_half2(v[2], v[6]), pack_half2(v[3], v[7]));
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(q_full(t));
            }
            int lo = 0, hi = 0;
            if (live) attn_range(a, p.r, i, lo, hi);
            // ref: a score, before its factor; rows that do not exist see nothing and need none
            float ref = live ? -INFINITY : 0.f, sum = 0.f, off = kTilePShift;
            bool far = false;
            for (int c = p.from; c < p.to; ++c) {
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(s_full(t), s_phase, abort_flag));
                if (!ok) break;
                s_phase ^= 1u;
                tc_fence_after();
                const int j0 = (p.range.chunk0 + c) * kTileKeys;
                const bool whole = j0 >= p.range.lo_all && j0 + kTileKeys <= p.range.hi_all;
                const float top = (whole ? tile_max<true>(s_tmem, 0, 0) : tile_max<false>(s_tmem, lo - j0, hi - j0));
                const bool move = top > ref && (top - ref) * mult > kTileSlack;             // infinite from -infinity
                if (__any_sync(0xffffffffu, move)) {
                    const float f = move ? exp2_approx((ref - top) * mult) : 1.f;             // 0 from -infinity
                    if (move) { ref = top; sum *= f; off = kTilePShift - top * mult; }
                    far = __any_sync(0xffffffffu, fabsf(off) > kTileFar);
                    if (c > p.from) {
#pragma unroll
                        for (int ch = 0; ch < HD / 16; ++ch) {
                            uint32_t r[16];
                            tc_ld16(o_tmem + ch * 16, r);
                            tc_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
                            tc_st16(o_tmem + ch * 16, r);
                        }
                    }
                }
                if (far) sum += tile_probs_far(s_tmem, mult, ref == -INFINITY ? 0.f : ref, whole ? 0 : lo - j0, whole ? kTileKeys : hi - j0);
                else sum += whole ? tile_probs<true>(s_tmem, mult, off, 0, 0) : tile_probs<false>(s_tmem, mult, off, lo - j0, hi - j0);
                tc_wait_st();
                tc_fence_before();
                mbar_arrive(p_full(t));
            }
            if (!ok) break;
            ok = __all_sync(0xffffffffu, mbar_wait_bounded(o_full(t), o_phase, abort_flag));
            if (!ok) break;
            o_phase ^= 1u;
            tc_fence_after();
            const bool complete = p.from == 0 && p.to == p.range.chunks;
            ref = ref == -INFINITY ? ref : ref * mult;
            const float inv = sum == 0.f ? 0.f : 1.f / sum, base_ref = ref == -INFINITY ? 0.f : ref;
            T* out = static_cast<T*>(a.out) + (int64_t)(p.r.row0 + i) * a.o_token + (int64_t)qh * a.o_head;
            float* slot = a.partial + (2 * blockIdx.x + (p.from == 0)) * tile_partial_floats(HD);
            const int in = t * 128 + row;
#pragma unroll
            for (int ch = 0; ch < HD / 16; ++ch) {
                uint32_t r[16];
                float v[16];
                tc_ld16(o_tmem + ch * 16, r);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = complete ? __uint_as_float(r[e]) * inv : __uint_as_float(r[e]);
                if (live && complete) store_row16<T>(out + ch * 16, v, 16, a.o_vec);
                if (live && !complete) store_row16<float>(slot + in * HD + ch * 16, v, 16, true);
            }
            if (live && complete && a.lse) a.lse[(int64_t)(p.r.row0 + i) * a.q_heads + qh] = attn_lse(base_ref, sum, kTilePShift);
            if (live && !complete) { slot[kTileRows * HD + in] = ref; slot[kTileRows * (HD + 1) + in] = sum; }
            tc_fence_before();                  // O has been read before this tile's next P is handed on
        }
        if (!ok && lane == 0) *abort_flag = 1;
    } else if (warp < 12) {
        // ------------------------------------------------------------ unpacking
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        constexpr int kK = HD / 32, kV = HD / 64;              // 16-byte pieces: a key; half a value
        const int u = threadIdx.x - 256, half = (warp - 8) & 1, dims = (warp - 8) >> 1, pair = half * 64 + 2 * lane;
        struct Raw { uint4 k[kK], v[2][kV]; uint32_t kg[kK / 2], vg[2]; } now, ahead;
        auto fetch = [&](const TilePiece& q, int c, Raw& x) {
            const int j0 = (q.range.chunk0 + c) * kTileKeys, per = a.cache.page_shift - 4;
            auto tile_of = [&](int j) -> const uint8_t* {
                const int tl = j >> 4;
                // no token there that any row sees: below the window there may be no page any more
                if (tl * kC4Tile >= q.range.hi_any || tl * kC4Tile + kC4Tile <= q.range.lo_any) return nullptr;
                int page = a.table[(int64_t)q.b * a.ldt + (tl >> per)];
                if (page < 0 || page >= a.cache.num_pages) { report(a.status, PTQ_ERR_INVALID_ARG, q.b, 2); page = 0; }
                return c4_tile<HD>(a.cache, page, q.head, tl & ((1 << per) - 1));
            };
            const uint8_t* kt = tile_of(j0 + u);
            const int kr = (j0 + u) & 15;
#pragma unroll
            for (int e = 0; e < kK; ++e) x.k[e] = kt ? ld_global16(kt + kr * (HD / 2) + 16 * e) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < kK / 2; ++e) x.kg[e] = kt ? ld_global4(kt + kCodes + kr * kGrids + 4 * e) : 0u;
            const uint8_t* vt = tile_of(j0 + pair);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = j0 + pair + h, vr = j & 15;
                const uint8_t* side = vt + kSide;
#pragma unroll
                for (int e = 0; e < kV; ++e)
                    x.v[h][e] = vt ? ld_global16(side + vr * (HD / 2) + dims * (HD / 4) + 16 * e) : make_uint4(0, 0, 0, 0);
                // what nobody sees may hold anything: 0 times it has to be 0
                const bool seen = vt && j >= q.range.lo_any && j < q.range.hi_any;
                if constexpr (HD == 128) x.vg[h] = seen ? ld_global4(side + kCodes + vr * kGrids + 4 * dims) : 0u;
                else x.vg[h] = seen ? ld_global2(side + kCodes + vr * kGrids + 2 * dims) : 0u;
            }
        };
        auto unpack = [&](unsigned char* stage, const Raw& x) {
            const uint32_t* kw = reinterpret_cast<const uint32_t*>(x.k);
#pragma unroll
            for (int g = 0; g < kK; ++g) {                     // groups of 32 values: four pieces of 16 bytes
                const uint32_t word = (x.kg[g >> 1] >> (16 * (g & 1))) & 0xffffu;
                const C4Factors f = c4_factors(word | word << 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t o[4];
                    c4_unpack4(kw[4 * g + e], kw[4 * g + e] >> 8, f, a.by, o);
                    *reinterpret_cast<uint4*>(stage + tile_at(kTileKeys, u, 4 * g + e)) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
            unsigned char* vt = stage + S::k_bytes + half * HD * 128;
#pragma unroll
            for (int g = 0; g < kV; ++g) {
                const C4Factors f = c4_factors(((x.vg[0] >> (16 * g)) & 0xffffu) | (x.vg[1] >> (16 * g)) << 16);
                const uint32_t *va = reinterpret_cast<const uint32_t*>(&x.v[0][g]), *vb = reinterpret_cast<const uint32_t*>(&x.v[1][g]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t o[4];
                        c4_unpack4(__byte_perm(va[e], vb[e], h ? 0x7632 : 0x5410), __byte_perm(va[e], vb[e], h ? 0x0703 : 0x0501), f, a.by, o);
#pragma unroll
                        for (int d = 0; d < 4; ++d) {
                            const int dim = dims * (HD / 2) + g * 32 + e * 8 + h * 4 + d;
                            *reinterpret_cast<uint32_t*>(vt + dim * 128 + (((lane >> 2) ^ (dim & 7)) << 4) + (lane & 3) * 4) = o[d];
                        }
                    }
            }
        };
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        while (ok && walk.next(a, list, p)) {
            fetch(p, p.from, ahead);
            for (int c = p.from; c < p.to; ++c) {
                now = ahead;
                if (c + 1 < p.to) fetch(p, c + 1, ahead);
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(kv_empty(stage), phase ^ 1u, abort_flag));
                if (!ok) break;
                unpack(base_ptr + S::q_bytes + stage * S::stage_bytes, now);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                mbar_arrive(kv_full(stage));
                if (++stage == 2) { stage = 0; phase ^= 1u; }
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 12) {
            // ------------------------------------------------------------ products
            int stage = 0;
            uint32_t kv_phase = 0, q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
            bool ok = true;
            auto scores = [&](int t, int st) {
                const uint32_t qa = kF8DescLo + ((base + t * (S::q_bytes / 2)) >> 4), kb = kF8DescLo + ((base + S::q_bytes + st * S::stage_bytes) >> 4);
#pragma unroll
                for (int ks = 0; ks < HD / 16; ++ks) {
                    const uint32_t at = (ks >> 2) * (128 * 128 >> 4) + (ks & 3) * 2;
                    tc_mma_f16(tmem + t * 128, qa + at, kb + at, f16_idesc(kTileKeys), ks > 0);
                }
                tc_commit_elected(s_full(t));
            };
            while (ok && walk.next(a, list, p)) {
                const bool two = p.r.n * a.ratio - p.tile * kTileRows > 128;
                const int tiles = two ? 2 : 1;
                ok = __all_sync(0xffffffffu, mbar_wait_bounded(kv_full(stage), kv_phase, abort_flag));
                for (int t = 0; t < tiles && ok; ++t) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(q_full(t), q_phase[t], abort_flag));
                    if (!ok) break;
                    q_phase[t] ^= 1u;
                    tc_fence_after();
                    scores(t, stage);
                }
                for (int c = p.from; c < p.to && ok; ++c) {
                    const int next = stage ^ 1;
                    const uint32_t next_phase = kv_phase ^ (stage == 1 ? 1u : 0u);
                    const bool more = c + 1 < p.to;
                    for (int t = 0; t < tiles; ++t) {
                        ok = __all_sync(0xffffffffu, mbar_wait_bounded(p_full(t), p_phase[t], abort_flag));
                        if (!ok) break;
                        p_phase[t] ^= 1u;
                        tc_fence_after();
                        const uint32_t vb = kF8DescLo + ((base + S::q_bytes + stage * S::stage_bytes + S::k_bytes) >> 4);
#pragma unroll
                        for (int ks = 0; ks < kTileKeys / 16; ++ks)
                            tc_mma_f16_tmem(tmem + 256 + t * 128, tmem + t * 128 + ks * 8, vb + (ks >> 2) * (HD * 128 >> 4) + (ks & 3) * 2, f16_idesc(HD),
                                            c > p.from || ks > 0);
                        if (t == tiles - 1) tc_commit_elected(kv_empty(stage));
                        if (more) {
                            if (t == 0) {
                                ok = __all_sync(0xffffffffu, mbar_wait_bounded(kv_full(next), next_phase, abort_flag));
                                if (!ok) break;
                                tc_fence_after();
                            }
                            scores(t, next);
                        } else {
                            tc_commit_elected(o_full(t));
                        }
                    }
                    stage = next;
                    kv_phase = next_phase;
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 12) {
        __syncwarp();
        tc_dealloc(tmem, 512u);
    }
    if (threadIdx.x == 0 && abort_word) report(a.status, PTQ_ERR_TIMEOUT, blockIdx.x, 4);
}

// Joins what CTAs share of a tile, as attn4_join_kernel does; a CTA takes one slice of the rows.
constexpr int kTileJoinSlices = 8;
template <typename T, int HD>
__global__ void __launch_bounds__(256) attn4_tile_join_kernel(Attn4 a, TileList list, int ctas) {
    constexpr int kLane = HD / 32;
    __shared__ int found;
    chained_begin();
    const int count = (int)list.before[list.most + 1], warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long total = a.cache.kv_heads * list.before[count], share = tile_share(total, ctas), u = share * (blockIdx.x + 1);
    if (u >= total) return;
    tile_find(a, list, count, u, &found);
    const int f = found;
    const long long length = list.before[f + 1] - list.before[f], rel = u - a.cache.kv_heads * list.before[f];
    const int head = (int)(rel / length);
    const long long end = a.cache.kv_heads * list.before[f] + (head + 1) * length, s0 = end - length + kTileCost;      // its first chunk
    if (s0 >= u) return;
    const int c0 = (int)(s0 / share), c1 = (int)((end - 1) / share);
    if (c0 != (int)blockIdx.x) return;
    const int2 at = list.tile[f];
    const AttnRows r = attn_rows(a, at.x);
    // four rows a warp side by side: their loads are in flight together
    constexpr int kJoin = kTileRows / kTileJoinSlices / 8;
    const int first = at.y * kTileRows, live = min(kTileRows, r.n * a.ratio - first), row0 = blockIdx.y * (kTileRows / kTileJoinSlices) + warp;
    float ref[kJoin], sum[kJoin], v[kJoin][kLane];
#pragma unroll
    for (int k = 0; k < kJoin; ++k) {
        ref[k] = -INFINITY;
        sum[k] = 0.f;
#pragma unroll
        for (int i = 0; i < kLane; ++i) v[k][i] = 0.f;
    }
    for (int c = c0; c <= c1; ++c) {
        const float* slot = a.partial + (2 * c + (c == c0)) * tile_partial_floats(HD);
#pragma unroll
        for (int k = 0; k < kJoin; ++k)
            if (row0 + 8 * k < live) ref[k] = fmaxf(ref[k], slot[kTileRows * HD + row0 + 8 * k]);
    }
#pragma unroll
    for (int k = 0; k < kJoin; ++k) ref[k] = ref[k] == -INFINITY ? 0.f : ref[k];
    for (int c = c0; c <= c1; ++c) {
        const float* slot = a.partial + (2 * c + (c == c0)) * tile_partial_floats(HD);
#pragma unroll
        for (int k = 0; k < kJoin; ++k) {
            const int row = row0 + 8 * k;
            if (row >= live) continue;
            const float w = exp2_approx(slot[kTileRows * HD + row] - ref[k]);
            sum[k] += w * slot[kTileRows * (HD + 1) + row];
#pragma unroll
            for (int i = 0; i < kLane; ++i) v[k][i] += w * slot[row * HD + lane * kLane + i];
        }
    }
#pragma unroll
    for (int k = 0; k < kJoin; ++k) {
        const int row = row0 + 8 * k;
        if (row >= live) continue;
        const int rr = first + row, i0 = rr / a.ratio, qh = head * a.ratio + rr - i0 * a.ratio;
        const float inv = sum[k] == 0.f ? 0.f : 1.f / sum[k];
        T* out = static_cast<T*>(a.out) + (int64_t)(r.row0 + i0) * a.o_token + (int64_t)qh * a.o_head + lane * kLane;
#pragma unroll
        for (int i = 0; i < kLane; ++i) out[i] = from_f32<T>(v[k][i] * inv);
        if (lane == 0 && a.lse) a.lse[(int64_t)(r.row0 + i0) * a.q_heads + qh] = attn_lse(ref[k], sum[k], kTilePShift);
    }
}

}  // namespace ptq
