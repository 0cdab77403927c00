// C-ABI entry points of the low-bit serving operators (see include/ptq.h): argument checks and the choice of kernels.
#include "attn4tile.cuh"
#include "cache4.cuh"
#include "common.cuh"
#include "fp8.cuh"

using namespace ptq;

namespace {

int type_size(int type) { return type == PTQ_F32 ? 4 : type == PTQ_F16 || type == PTQ_BF16 ? 2 : 0; }

// Calls f with a null pointer of the type that `type` names.
template <typename F>
int with_type(int type, F f) {
    switch (type) {
        case PTQ_F32: return f(static_cast<float*>(nullptr));
        case PTQ_F16: return f(static_cast<__half*>(nullptr));
        case PTQ_BF16: return f(static_cast<__nv_bfloat16*>(nullptr));
    }
    return PTQ_ERR_INVALID_ARG;
}

// Whether an output's bytes [a, a + na) touch an input's (or another output's) [b, b + nb).
struct Span { const void* p; size_t n; };
bool touch(Span a, Span b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return a.p && b.p && a.n && b.n && x < y + b.n && y < x + a.n;
}
template <typename... S>
bool touch_any(Span a, S... others) { return (touch(a, others) || ...); }
Span rows_span(const void* p, int64_t rows, int64_t ld, int64_t cols, int size) {
    return {p, rows > 0 ? (size_t)((rows - 1) * ld + cols) * size : 0};
}
Span heads_span(const void* p, int64_t tokens, int64_t ld_token, int64_t heads, int64_t ld_head, int64_t dim, int size) {
    return {p, tokens > 0 ? (size_t)((tokens - 1) * ld_token + (heads - 1) * ld_head + dim) * size : 0};
}
// Whether two sets of rows [tokens][heads] of `width` bytes with the same strides (of at least that), the second `d` bytes behind
// the first, share a byte; `self`: whether two different rows of one set do.
bool rows_meet(int64_t d, int64_t tokens, int64_t heads, int64_t by_token, int64_t by_head, int64_t width, bool self) {
    if (self && (by_token >= (heads - 1) * by_head + width || by_head >= (tokens - 1) * by_token + width)) return false;      // one inside the other
    for (int64_t j = -(heads - 1); j <= heads - 1; ++j) {
        const int64_t x = d + j * by_head;                // row i of the second set begins x + i by_token behind some row of the first
        const int64_t down = -(x / by_token) - (x % by_token > 0);
        for (int64_t i = down; i <= down + 1; ++i) {
            const int64_t gap = x + i * by_token;
            if (i > -tokens && i < tokens && gap > -width && gap < width && !(self && i == 0 && j == 0)) return true;
        }
    }
    return false;
}
struct Rows { const void* p; int64_t tokens, by_token, heads, by_head, dim; int size; };
Span span_of(const Rows& r) { return heads_span(r.p, r.tokens, r.by_token, r.heads, r.by_head, r.dim, r.size); }
bool meets_itself(const Rows& r) { return rows_meet(0, r.tokens, r.heads, r.by_token * r.size, r.by_head * r.size, r.dim * r.size, true); }
// Rows of one shape may alternate in a buffer (the parts of a fused projection); with other strides whole spans are compared.
bool meet(const Rows& a, const Rows& b) {
    if (!touch(span_of(a), span_of(b))) return false;
    if (a.by_token != b.by_token || a.by_head != b.by_head || a.heads != b.heads || a.size != b.size || b.by_token < b.dim) return true;
    return rows_meet(static_cast<const char*>(b.p) - static_cast<const char*>(a.p), a.tokens, a.heads, a.by_token * a.size, a.by_head * a.size,
                     a.dim * a.size, false);
}

int page_shift_of(int page_size) {
    for (int s = 4; s <= 10; ++s)
        if (page_size == 1 << s) return s;
    return -1;
}

template <typename T, int NT>
cudaError_t allow_few_smem() {
    return cudaFuncSetAttribute(f8_product_few_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, F8Few<NT>::smem_bytes);
}
template <typename T>
cudaError_t allow_f8_smem() {
    cudaError_t e = cudaFuncSetAttribute(f8_product_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kF8SmemBytes);
    if (e == cudaSuccess) e = allow_few_smem<T, 16>();
    if (e == cudaSuccess) e = allow_few_smem<T, 32>();
    if (e == cudaSuccess) e = allow_few_smem<T, 64>();
    return e;
}

template <typename T, int NT>
int f8_few_launch(const F8Product& p, const uint8_t* A, int64_t lda, const uint8_t* B, int64_t ldb, int ks, cudaStream_t stream) {
    CUtensorMap mapA, mapB;
    int st = f8_map(&mapA, A, p.m, p.k, lda, NT);
    if (!st) st = f8_map(&mapB, B, p.n, p.k, ldb, 128);
    if (st) return st;
    Launch l(K_F8_PRODUCT_FEW, stream);
    launch_chained_cluster(f8_product_few_kernel<T, NT>, dim3(ks, cdiv(p.n, 128), cdiv(p.m, NT)), ks, kF8FewThreads,
                           F8Few<NT>::smem_bytes, stream, mapA, mapB, p, ks);
    return PTQ_OK;
}

// Which kernel, how many rows of A a tile holds and how many CTAs share a tile's k blocks.  Measured, us (bf16 results, operands from
// memory), rows a tile / CTAs a tile, `many` the persistent kernel:
//   1 x 4096 x 4096: 16/1 9.3, 16/4 6.2, 16/8 6.7;  16 x 4096 x 11008: 16/1 24.1, 16/4 13.3, 16/8 12.4;  1 x 11008 x 4096: 16/1 12.3, 16/4 14.9
//   64 x 4096 x 4096: 64/1 16.4, 64/4 11.8, 64/8 10.9;  333 x 1000 x 2048: 64/1 10.4, 64/4 11.7, 128/1 14.9, many 12.9
//   333 x 4096 x 4096: 64/1 21.3, 64/4 37, 128/1 24.7, many 21.1;  1000 x 2048 x 2048: 64/1 13.9, many 12.9;  2048 x 4096 x 4096: 81, many 41.1
// So: k is shared by four or eight CTAs while all of them are on the GPU at once (two an SM) and each keeps eight blocks, or four where
// one an SM is enough (two CTAs a tile were slower than either one or four); tiles of more than 64 rows never pay; and the
// persistent kernel takes over above them where its tiles fill two fifths of the SMs.
template <typename T>
int f8_launch(const F8Product& p, const uint8_t* A, int64_t lda, const uint8_t* B, int64_t ldb, int sms, cudaStream_t stream) {
    const long tiles_m = cdiv(p.m, kF8TileM), tiles_n = cdiv(p.n, kF8TileN);
    if (p.m > 64 && 5 * tiles_m * tiles_n >= 2 * sms) {
        CUtensorMap mapA, mapB;
        int st = f8_map(&mapA, A, p.m, p.k, lda, kF8TileM);
        if (!st) st = f8_map(&mapB, B, p.n, p.k, ldb, kF8TileN);
        if (st) return st;
        const int grid = (int)(tiles_m * tiles_n < sms ? tiles_m * tiles_n : sms);
        Launch l(K_F8_PRODUCT, stream);
        launch_chained(f8_product_kernel<T>, grid, kF8Threads, kF8SmemBytes, stream, mapA, mapB, p, (int)tiles_m, (int)tiles_n);
        return PTQ_OK;
    }
    const int nt = p.m <= 16 ? 16 : p.m <= 32 ? 32 : 64;
    const long tiles = (long)cdiv(p.n, 128) * cdiv(p.m, nt);
    int ks = 1;
    for (int c = 4; c <= 8; c *= 2)
        if ((tiles * c <= 2 * sms && p.kb >= 8 * c) || (tiles * c <= sms && p.kb >= 4 * c)) ks = c;
    switch (nt) {
        case 16: return f8_few_launch<T, 16>(p, A, lda, B, ldb, ks, stream);
        case 32: return f8_few_launch<T, 32>(p, A, lda, B, ldb, ks, stream);
    }
    return f8_few_launch<T, 64>(p, A, lda, B, ldb, ks, stream);
}

int cache_check(Cache4* c, const void* pages, int num_pages, int page_size, int kv_heads, int head_dim) {
    const int shift = page_shift_of(page_size);
    if (!pages || num_pages < 1 || kv_heads < 1 || head_dim < 1) return PTQ_ERR_INVALID_ARG;
    if (shift < 0 || (head_dim != 64 && head_dim != 128) || kv_heads > 65535) return PTQ_ERR_UNSUPPORTED;
    if ((int64_t)num_pages * page_size > 0x7fffffffll) return PTQ_ERR_UNSUPPORTED;       // slots are int32
    if (!aligned16(pages)) return PTQ_ERR_ALIGNMENT;
    c->pages = static_cast<uint8_t*>(const_cast<void*>(pages));
    c->num_pages = num_pages;
    c->page_shift = shift;
    c->kv_heads = kv_heads;
    return PTQ_OK;
}

bool rows_aligned(const void* p, int64_t a, int64_t b, int size) { return aligned16(p) && a * size % 16 == 0 && b * size % 16 == 0; }

// Append and read share their arguments.
int cache_tokens(bool append, const Cache4& c, int head_dim, C4Tokens a, int type, cudaStream_t stream) {
    a.vec = rows_aligned(a.k, a.k_token, a.k_head, type_size(type)) && rows_aligned(a.v, a.v_token, a.v_head, type_size(type));
    const int64_t threads = (int64_t)a.tokens * c.kv_heads * 2 * (head_dim / 8), grid = (threads + 255) / 256;
    if (grid > 0x7fffffffll) return PTQ_ERR_UNSUPPORTED;
    return with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        Launch l(append ? K_CACHE_APPEND : K_CACHE_READ, stream);
        if (append) {
            if (head_dim == 128) launch_chained(cache_append_kernel<T, 128>, (unsigned)grid, 256, 0, stream, c, a);
            else launch_chained(cache_append_kernel<T, 64>, (unsigned)grid, 256, 0, stream, c, a);
        } else {
            if (head_dim == 128) launch_chained(cache_read_kernel<T, 128>, (unsigned)grid, 256, 0, stream, c, a);
            else launch_chained(cache_read_kernel<T, 64>, (unsigned)grid, 256, 0, stream, c, a);
        }
        return launch_status();
    });
}

template <typename T, int HD, int NT>
cudaError_t allow_attn_smem() {
    return cudaFuncSetAttribute(attn4_few_kernel<T, HD, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewShape<HD, NT>::smem_bytes);
}
template <typename T>
cudaError_t allow_attn_smem_all() {
    cudaError_t e = allow_attn_smem<T, 64, 1>();
    if (e == cudaSuccess) e = allow_attn_smem<T, 64, 2>();
    if (e == cudaSuccess) e = allow_attn_smem<T, 128, 1>();
    if (e == cudaSuccess) e = allow_attn_smem<T, 128, 2>();
    if (e == cudaSuccess) e = cudaFuncSetAttribute(attn4_tile_kernel<T, 64>, cudaFuncAttributeMaxDynamicSharedMemorySize, TileShape<64>::smem_bytes);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(attn4_tile_kernel<T, 128>, cudaFuncAttributeMaxDynamicSharedMemorySize, TileShape<128>::smem_bytes);
    return e;
}

template <typename T, int HD, int NT>
void attn_few_launch(const Attn4& a, int sms, cudaStream_t stream) {
    using F = FewShape<HD, NT>;
    const int ctas = sms < kFewMaxCtas ? sms : kFewMaxCtas;
    {
        Launch l(K_CACHE_ATTN_FEW, stream);
        launch_chained(attn4_few_kernel<T, HD, NT>, ctas, F::threads, F::smem_bytes, stream, a);
    }
    {
        Launch l(K_CACHE_ATTN_JOIN, stream);
        launch_chained(attn4_join_kernel<T, HD, NT>, cdiv(ctas * F::warps, kJoinWarps), kJoinThreads, 0, stream, a, ctas);
    }
}
template <typename T, int HD>
void attn_tile_launch(const Attn4& a, const TileList& list, int sms, cudaStream_t stream) {
    const int ctas = sms < kTileMaxCtas ? sms : kTileMaxCtas;
    {
        Launch l(K_CACHE_ATTN_SCHEDULE, stream);
        launch_chained(attn4_schedule_kernel, 1, kScheduleThreads, 0, stream, a, list);
    }
    {
        Launch l(K_CACHE_ATTN_TILE, stream);
        launch_chained(attn4_tile_kernel<T, HD>, ctas, kTileThreads, TileShape<HD>::smem_bytes, stream, a, list);
    }
    {
        Launch l(K_CACHE_ATTN_TILE_JOIN, stream);
        launch_chained(attn4_tile_join_kernel<T, HD>, dim3(ctas - 1, kTileJoinSlices), 256, 0, stream, a, list, ctas);
    }
}

// Requests with up to this many rows (new tokens x query heads of a kv head) go to the kernel for few rows, others to the tiles.  Measured
// with heads of 128, us, few rows / tiles, by rows of a request:
//   64 requests of up to 2048 tokens, 4 kv heads:  16: 63 / 82;  24: 92 / 82;  32: 98 / 82;  64: 168 / 85;  128: 297 / 90
//   8 requests of up to 8192 tokens, 8 kv heads:   16: 69 / 68;  24: 69 / 70;  32: 74 / 71;  64: 112 / 73;  128: 191 / 78
//   1 request of 8192 tokens, 8 kv heads:          16: 85 / 41;  24: 61 / 45;  32: 64 / 50;  64: 63 / 52;   128: 69 / 55
// A request alone is split so finely that joining its parts costs the kernel for few rows as much as the attention does; batches decide.
constexpr int kFewRows = 16;

// The pieces of attention's workspace.
struct AttnSpace {
    float *few, *tiles;
    TileList list;
    size_t bytes;
};
AttnSpace attn_space(void* ws, int ratio, int head_dim, int batch, int total_q, int max_q) {
    AttnSpace s{};
    Carver cv(ws);
    const int64_t rows = (int64_t)max_q * ratio;
    const int nt = rows <= 8 ? 1 : 2;
    s.few = cv.take<float>((size_t)2 * kFewMaxCtas * few_warps(nt) * few_partial_floats(head_dim, nt));
    if (rows > kFewRows) {
        s.tiles = cv.take<float>((size_t)2 * kTileMaxCtas * tile_partial_floats(head_dim));
        s.list.most = (int)((int64_t)total_q * ratio / kTileRows) + batch;           // a last, partly filled tile for each request
        s.list.before = cv.take<long long>((size_t)s.list.most + 2);
        s.list.tile = cv.take<int2>((size_t)s.list.most);
    }
    s.bytes = cv.off;
    return s;
}

template <typename T, int HD>
int attn_launch(Attn4 a, const AttnSpace& space, int max_q, int sms, cudaStream_t stream) {
    const int64_t rows = (int64_t)max_q * a.ratio;
    a.partial = space.few;
    if (rows <= kFewRows) {
        a.row_limit = 0x7fffffff;
        if (rows <= 8) attn_few_launch<T, HD, 1>(a, sms, stream);
        else attn_few_launch<T, HD, 2>(a, sms, stream);
        return launch_status();
    }
    // where every request has max_q rows there are none with few
    a.row_limit = (int64_t)max_q * a.batch == a.total_q ? 0 : kFewRows;
    if (a.row_limit > 0) attn_few_launch<T, HD, 2>(a, sms, stream);
    a.partial = space.tiles;
    attn_tile_launch<T, HD>(a, space.list, sms, stream);
    return launch_status();
}

}  // namespace

extern "C" {

int ptq_fp8_quantize(const void* x, int x_type, int rows, int cols, int64_t ldx, int block_rows, uint8_t* q, int64_t ldq, float* scale,
                     int64_t ld_scale, int32_t* status, void* stream_) {
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int size = type_size(x_type), kb = cols > 0 ? cdiv(cols, kF8Block) : 0;
    if (rows < 0 || cols < 1 || !size || (block_rows != 1 && block_rows != kF8Block)) return PTQ_ERR_INVALID_ARG;
    if (rows == 0) return PTQ_OK;
    if (!x || !q || !scale || ldx < cols || ldq < cols || ld_scale < kb) return PTQ_ERR_INVALID_ARG;
    if (rows > 0x7fffff00 || cols > 0x7fffff00 || (block_rows > 1 ? cdiv(rows, kF8Block) : cdiv(kb, 2)) > 65535) return PTQ_ERR_UNSUPPORTED;
    if (!aligned16(q) || (rows > 1 && ldq % 16)) return PTQ_ERR_ALIGNMENT;
    const Span in = rows_span(x, rows, ldx, cols, size), codes = rows_span(q, rows, ldq, cols, 1),
               factors = rows_span(scale, cdiv(rows, block_rows), ld_scale, kb, 4);
    if (touch_any(codes, in, factors) || touch(factors, in)) return PTQ_ERR_INVALID_ARG;
    const int vec = aligned16(x) && ldx * size % 16 == 0;
    return with_type(x_type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const T* xs = static_cast<const T*>(x);
        if (block_rows == 1) {
            Launch l(K_F8_QUANTIZE, stream);
            launch_chained(f8_quantize_rows_kernel<T>, dim3((rows - 1) / 8 + 1, cdiv(kb, 2)), 256, 0, stream, xs, rows, cols, ldx, vec, q, ldq, scale, ld_scale,
                           status);
        } else {
            Launch l(K_F8_QUANTIZE, stream);
            launch_chained(f8_quantize_blocks_kernel<T>, dim3(kb, cdiv(rows, kF8Block)), 256, 0, stream, xs, rows, cols, ldx, vec, q, ldq,
                           scale, ld_scale, status);
        }
        return launch_status();
    });
}

int ptq_fp8_matmul(void* C, int c_type, int64_t ldc, const uint8_t* A, int64_t lda, const float* scale_a, int64_t ld_scale_a,
                   const uint8_t* B, int64_t ldb, const float* scale_b, int64_t ld_scale_b, int m, int n, int k, int32_t* status,
                   void* stream_) {
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int kb = k > 0 ? cdiv(k, kF8Block) : 0;
    if (m < 0 || n < 0 || k < 1 || !type_size(c_type)) return PTQ_ERR_INVALID_ARG;
    if (m == 0 || n == 0) return PTQ_OK;
    if (!C || !A || !B || !scale_a || !scale_b || ldc < n || lda < k || ldb < k || ld_scale_a < kb || ld_scale_b < kb)
        return PTQ_ERR_INVALID_ARG;
    if (k > 0x7fffff00 || m > 1 << 20 || n > 1 << 22) return PTQ_ERR_UNSUPPORTED;
    if (m == 1) lda = ((int64_t)k + 15) / 16 * 16;       // the stride of a single row is never used, but a tensor map has one
    if (n == 1) ldb = ((int64_t)k + 15) / 16 * 16;
    if (!aligned16(A) || !aligned16(B) || lda % 16 || ldb % 16) return PTQ_ERR_ALIGNMENT;
    if (touch_any(rows_span(C, m, ldc, n, type_size(c_type)), rows_span(A, m, lda, k, 1), rows_span(B, n, ldb, k, 1),
                  rows_span(scale_a, m, ld_scale_a, kb, 4), rows_span(scale_b, cdiv(n, kF8Block), ld_scale_b, kb, 4)))
        return PTQ_ERR_INVALID_ARG;
    DeviceState* dev = nullptr;
    int st = current_device_state(&dev);
    if (st) return st;
    st = ensure_smem_attr(dev, SA_F8_PRODUCT, [] {
        cudaError_t e = allow_f8_smem<float>();
        if (e == cudaSuccess) e = allow_f8_smem<__half>();
        if (e == cudaSuccess) e = allow_f8_smem<__nv_bfloat16>();
        return e;
    });
    if (st) return st;
    F8Product p{C, scale_a, scale_b, ldc, ld_scale_a, ld_scale_b, m, n, k, kb, status};
    st = with_type(c_type, [&](auto* t) { return f8_launch<std::remove_pointer_t<decltype(t)>>(p, A, lda, B, ldb, dev->sms, stream); });
    return st ? st : launch_status();
}

size_t ptq_cache_page_bytes(int page_size, int kv_heads, int head_dim) {
    if (page_shift_of(page_size) < 0 || kv_heads < 1 || kv_heads > 65535 || (head_dim != 64 && head_dim != 128)) return 0;
    return (size_t)kv_heads * (page_size / kC4Tile) * c4_tile_bytes(head_dim);
}

int ptq_cache_plan(const int32_t* kv_lens, const int32_t* new_tokens, int batch, int page_size, int32_t* block_table, int64_t ld_table,
                   int max_pages, const int32_t* free_pages, int num_free, int32_t* slots, int32_t* positions, int max_tokens,
                   int32_t* cu_q, int32_t* kv_lens_out, int32_t* taken, int32_t* status, void* stream_) {
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const int shift = page_shift_of(page_size);
    if (batch < 0 || max_pages < 0 || ld_table < max_pages || num_free < 0 || max_tokens < 0 || !cu_q || !taken) return PTQ_ERR_INVALID_ARG;
    if (batch > 0 && (!kv_lens || !new_tokens || !kv_lens_out || (max_pages > 0 && !block_table))) return PTQ_ERR_INVALID_ARG;
    if ((num_free > 0 && !free_pages) || (max_tokens > 0 && (!slots || !positions))) return PTQ_ERR_INVALID_ARG;
    const size_t per_request = (size_t)batch * 4, per_token = (size_t)max_tokens * 4;
    const Span lens{kv_lens, per_request}, fresh{new_tokens, per_request}, pages{free_pages, (size_t)num_free * 4},
        table = rows_span(block_table, max_pages > 0 ? batch : 0, ld_table, max_pages, 4), at{slots, per_token}, pos{positions, per_token},
        cu{cu_q, per_request + 4}, after{kv_lens_out, per_request}, count{taken, 4};
    if (touch_any(table, lens, fresh, pages, at, pos, cu, after, count) || touch_any(at, lens, fresh, pages, pos, cu, after, count) ||
        touch_any(pos, lens, fresh, pages, cu, after, count) || touch_any(cu, lens, fresh, pages, after, count) ||
        touch_any(after, lens, fresh, pages, count) || touch_any(count, lens, fresh, pages))
        return PTQ_ERR_INVALID_ARG;                     // every CTA reads what one of them writes for all
    if (shift < 0 || (int64_t)max_pages * page_size > (1ll << 30)) return PTQ_ERR_UNSUPPORTED;
    CachePlan p{kv_lens, new_tokens, batch, block_table, ld_table, max_pages, free_pages, num_free, shift, slots, positions, max_tokens,
                cu_q, kv_lens_out, taken, status};
    const int grid = max_tokens > kPlanTokens ? (int)(((int64_t)max_tokens + kPlanTokens - 1) / kPlanTokens) : 1;
    Launch l(K_CACHE_PLAN, stream);
    launch_chained(cache_plan_kernel, grid, kPlanThreads, 0, stream, p);
    return launch_status();
}

int ptq_cache_append(void* pages, int num_pages, int page_size, int kv_heads, int head_dim, const void* k, int64_t k_token, int64_t k_head,
                     const void* v, int64_t v_token, int64_t v_head, int type, const int32_t* slots, int tokens, int32_t* status,
                     void* stream_) {
    Cache4 c;
    const int st = cache_check(&c, pages, num_pages, page_size, kv_heads, head_dim);
    if (st) return st;
    if (tokens < 0 || !type_size(type)) return PTQ_ERR_INVALID_ARG;
    if (tokens == 0) return PTQ_OK;
    if (!k || !v || !slots || k_token < 0 || k_head < 0 || v_token < 0 || v_head < 0) return PTQ_ERR_INVALID_ARG;
    const Span all{pages, (size_t)num_pages * ptq_cache_page_bytes(page_size, kv_heads, head_dim)}, at{slots, (size_t)tokens * 4};
    if (touch_any(all, heads_span(k, tokens, k_token, kv_heads, k_head, head_dim, type_size(type)),
                  heads_span(v, tokens, v_token, kv_heads, v_head, head_dim, type_size(type)), at))
        return PTQ_ERR_INVALID_ARG;
    return cache_tokens(true, c, head_dim,
                        C4Tokens{const_cast<void*>(k), const_cast<void*>(v), k_token, k_head, v_token, v_head, slots, tokens, 0, status},
                        type, static_cast<cudaStream_t>(stream_));
}

int ptq_cache_read(const void* pages, int num_pages, int page_size, int kv_heads, int head_dim, void* k, int64_t k_token, int64_t k_head,
                   void* v, int64_t v_token, int64_t v_head, int type, const int32_t* slots, int tokens, int32_t* status, void* stream_) {
    Cache4 c;
    const int st = cache_check(&c, pages, num_pages, page_size, kv_heads, head_dim);
    if (st) return st;
    if (tokens < 0 || !type_size(type)) return PTQ_ERR_INVALID_ARG;
    if (tokens == 0) return PTQ_OK;
    if (!k || !v || !slots || k_token < head_dim || k_head < head_dim || v_token < head_dim || v_head < head_dim) return PTQ_ERR_INVALID_ARG;
    const Span all{pages, (size_t)num_pages * ptq_cache_page_bytes(page_size, kv_heads, head_dim)}, at{slots, (size_t)tokens * 4};
    const Rows kr{k, tokens, k_token, kv_heads, k_head, head_dim, type_size(type)}, vr{v, tokens, v_token, kv_heads, v_head, head_dim, type_size(type)};
    if (touch_any(span_of(kr), all, at) || touch_any(span_of(vr), all, at) || meets_itself(kr) || meets_itself(vr) || meet(kr, vr))
        return PTQ_ERR_INVALID_ARG;
    return cache_tokens(false, c, head_dim, C4Tokens{k, v, k_token, k_head, v_token, v_head, slots, tokens, 0, status}, type,
                        static_cast<cudaStream_t>(stream_));
}

size_t ptq_cache_attention_workspace_bytes(int q_heads, int kv_heads, int head_dim, int batch, int total_q, int max_q) {
    if (q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || batch < 0 || total_q < 0 || max_q < 0 || (head_dim != 64 && head_dim != 128) ||
        (int64_t)total_q * q_heads > 0x7fffffffll)
        return 0;
    return attn_space(nullptr, q_heads / kv_heads, head_dim, batch, total_q, max_q).bytes;
}

int ptq_cache_attention(void* out, int64_t o_token, int64_t o_head, float* lse, const void* q, int64_t q_token, int64_t q_head, int type,
                        int q_heads, const void* pages, int num_pages, int page_size, int kv_heads, int head_dim,
                        const int32_t* block_table, int64_t ld_table, int max_pages, const int32_t* kv_lens, const int32_t* cu_q,
                        int batch, int total_q, int max_q, float scale, int causal, int window, void* ws, size_t ws_bytes,
                        int32_t* status, void* stream_) {
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    Attn4 a{};
    int st = cache_check(&a.cache, pages, num_pages, page_size, kv_heads, head_dim);
    if (st) return st;
    if (q_heads < 1 || q_heads % kv_heads || batch < 0 || total_q < 0 || max_q < 0 || max_pages < 0 || ld_table < max_pages || window < 0 ||
        (causal != 0 && causal != 1) || (type != PTQ_F16 && type != PTQ_BF16) || !(fabsf(scale) <= 2.0e38f))
        return PTQ_ERR_INVALID_ARG;
    if (batch == 0 || total_q == 0 || max_q == 0) return PTQ_OK;
    if (!out || !q || !kv_lens || !cu_q || (max_pages > 0 && !block_table) || o_token < head_dim || o_head < head_dim || q_token < 0 || q_head < 0)
        return PTQ_ERR_INVALID_ARG;
    if ((int64_t)max_pages * page_size > (1ll << 30) || (int64_t)total_q * q_heads > 0x7fffffffll) return PTQ_ERR_UNSUPPORTED;
    if (!aligned16(ws)) return PTQ_ERR_ALIGNMENT;
    if (!ws || ws_bytes < ptq_cache_attention_workspace_bytes(q_heads, kv_heads, head_dim, batch, total_q, max_q)) return PTQ_ERR_WORKSPACE;
    const Rows orows{out, total_q, o_token, q_heads, o_head, head_dim, 2}, qrows{q, total_q, q_token, q_heads, q_head, head_dim, 2};
    const Span result = span_of(orows), sums{lse, (size_t)total_q * q_heads * 4},
               scratch{ws, ptq_cache_attention_workspace_bytes(q_heads, kv_heads, head_dim, batch, total_q, max_q)}, rows = span_of(qrows),
               all{pages, (size_t)num_pages * ptq_cache_page_bytes(page_size, kv_heads, head_dim)},
               table = rows_span(block_table, max_pages > 0 ? batch : 0, ld_table, max_pages, 4), lens{kv_lens, (size_t)batch * 4},
               cu{cu_q, (size_t)batch * 4 + 4};
    if (meet(orows, qrows) || meets_itself(orows) || touch_any(result, sums, scratch, all, table, lens, cu) || touch_any(sums, scratch, rows, all, table, lens, cu) ||
        touch_any(scratch, rows, all, table, lens, cu))
        return PTQ_ERR_INVALID_ARG;
    DeviceState* dev = nullptr;
    st = current_device_state(&dev);
    if (st) return st;
    st = ensure_smem_attr(dev, SA_CACHE_ATTN, [] {
        const cudaError_t e = allow_attn_smem_all<__half>();
        return e == cudaSuccess ? allow_attn_smem_all<__nv_bfloat16>() : e;
    });
    if (st) return st;
    a.q = q; a.out = out; a.lse = lse;
    a.q_token = q_token; a.q_head = q_head; a.o_token = o_token; a.o_head = o_head;
    a.table = block_table; a.ldt = ld_table; a.max_pages = max_pages; a.lens = kv_lens; a.cu = cu_q;
    a.batch = batch; a.total_q = total_q; a.q_heads = q_heads; a.ratio = q_heads / kv_heads;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.causal = causal; a.window = window;
    a.q_vec = rows_aligned(q, q_token, q_head, 2); a.o_vec = rows_aligned(out, o_token, o_head, 2);
    a.by = make_uint2(64u, 4u);
    a.status = status;
    const AttnSpace space = attn_space(ws, a.ratio, head_dim, batch, total_q, max_q);
    auto launch = [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return head_dim == 64 ? attn_launch<T, 64>(a, space, max_q, dev->sms, stream) : attn_launch<T, 128>(a, space, max_q, dev->sms, stream);
    };
    return type == PTQ_F16 ? launch(static_cast<__half*>(nullptr)) : launch(static_cast<__nv_bfloat16*>(nullptr));
}

}  // extern "C"
