// Operands in 8-bit floating point (e4m3) with one scale for each block of 128 values, and their product.
//
// Cast: the scale of a block is s = 2^e with the least e >= -126 that gives max |x| <= 448 s.  A power of two costs at most one
// of the format's binades and no precision (the format is a floating one), and x / s is then exact, so that a code is ONE
// rounding of x and the same wherever it is computed.
//
// Product: C[i][j] = sum_b sa[i][b] sb[j / 128][b] sum_{k in block b} A[i][k] B[j][k].  The scales change from block to block of k,
// so the tensor cores sum one block (4 steps of 32) into TMEM and the blocks are joined in float32 registers: acc += s d.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "tc.cuh"

namespace ptq {

constexpr int kF8Block = 128;

// ------------------------------------------------------------------------------------------------------------
// Values of 16 or 32 bits, eight at a time
// ------------------------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32(float x) { return x; }
template <> __device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32(float x) { return x; }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }

// Eight consecutive values of which `n` exist (the others become 0); vec: p is 16-byte aligned.  Plain loads, here and in all kernels of
// this kind: they are put in place while the kernel before them may still write what they read (chained_begin), and the read-only
// path (__ldg, const __restrict__) is for memory that nobody writes while a kernel lives.  Times are the same.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, bool vec, float (&v)[8]) {
    if (vec && n >= 8) {
        alignas(16) T t[8];
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(t)[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f32<T>(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32<T>(p[i]) : 0.f;
    }
}

// Two float32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
        "l"(*reinterpret_cast<unsigned long long*>(&c)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
    return *reinterpret_cast<float2*>(&r);
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// The larger magnitude; a NaN stays one (and an infinity is larger than anything else), so one look at the result tells.
__device__ __forceinline__ float max_magnitude(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
}

// Exponent e of the scale of a block whose largest magnitude is `top`: 448 = 1.75 2^8, so the mantissa of top decides by 1.75.
__device__ __forceinline__ int f8_exponent(float top) {
    const int e = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 127 - 8;
    return e < -126 ? -126 : e;
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }      // -126 <= e <= 127

// Two values to two codes, rounded to nearest even (nothing saturates: |x| <= 448).
__device__ __forceinline__ uint32_t f8_pair(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint2 f8_codes8(const float (&v)[8], float inv) {
    uint2 r;
    r.x = f8_pair(v[0] * inv, v[1] * inv) | f8_pair(v[2] * inv, v[3] * inv) << 16;
    r.y = f8_pair(v[4] * inv, v[5] * inv) | f8_pair(v[6] * inv, v[7] * inv) << 16;
    return r;
}
__device__ __forceinline__ void f8_store8(uint8_t* p, int n, uint2 c) {
    if (n >= 8) {
        *reinterpret_cast<uint2*>(p) = c;
    } else {
        for (int i = 0; i < n; ++i) p[i] = (uint8_t)((i < 4 ? c.x >> (8 * i) : c.y >> (8 * (i - 4))));
    }
}
constexpr uint32_t kF8NanCodes = 0x7f7f7f7fu;

// One scale per row and block of 128 columns: sixteen lanes hold a block, eight values each.  One read of x, one write of the codes;
// 16-bit inputs are bound by the instructions between them (8192 x 4096: float32 29 us, 5.7 TB/s; bf16 25 us, 4.1 TB/s).  A block a half warp: two or four
// in a row were slower (26.8, 30.8, 33.4 us with one, two, four).
template <typename T>
__global__ void __launch_bounds__(256) f8_quantize_rows_kernel(const T* x, int rows, int cols, int64_t ldx, int vec,
                                                                uint8_t* q, int64_t ldq, float* scale,
                                                                int64_t lds, int32_t* status) {
    chained_begin();
    // two blocks of eight rows: a warp's two half warps take neighbouring blocks
    const int blk = 2 * blockIdx.y + ((threadIdx.x >> 4) & 1), c0 = blk * kF8Block + (threadIdx.x & 15) * 8;
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= rows || blk * kF8Block >= cols) return;    // the lanes of a half warp stay or leave together
    const unsigned half = 0xffffu << (threadIdx.x & 16);
    float v[8], top = 0.f;
    load8<T>(x + row * ldx + c0, cols - c0, vec, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max_magnitude(top, v[j]);
#pragma unroll
    for (int s = 8; s > 0; s >>= 1) top = max_magnitude(top, __shfl_xor_sync(half, top, s));
    const bool bad = not_finite(top);
    const int e = f8_exponent(top);
    uint2 codes = f8_codes8(v, bad ? 0.f : exp2_int(-e));
    if (bad) codes = make_uint2(kF8NanCodes, kF8NanCodes);
    f8_store8(q + row * ldq + c0, cols - c0, codes);
    if ((threadIdx.x & 15) == 0) {
        scale[row * lds + blk] = bad ? __uint_as_float(0x7fc00000u) : exp2_int(e);
        if (bad) report(status, PTQ_ERR_NONFINITE, (int)row);
    }
}

// One scale per block of 128 x 128: a CTA holds the block in registers (64 values a thread), so x is read once.  4096 x 11008: float32 39 us
// (5.8 TB/s); bf16 and fp16 66 us (2.0 TB/s), bound by latency: sixteen warps an SM, and a thread's eight loads follow one another.
template <typename T>
__global__ void __launch_bounds__(256) f8_quantize_blocks_kernel(const T* x, int rows, int cols, int64_t ldx, int vec,
                                                                  uint8_t* q, int64_t ldq, float* scale,
                                                                  int64_t lds, int32_t* status) {
    chained_begin();
    __shared__ float warp_top[8];
    const int c0 = blockIdx.x * kF8Block + (threadIdx.x & 15) * 8, r0 = blockIdx.y * kF8Block + (threadIdx.x >> 4);
    float v[8][8], top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        load8<T>(x + (int64_t)(r < rows ? r : 0) * ldx + c0, r < rows ? cols - c0 : 0, vec, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max_magnitude(top, v[i][j]);
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) top = max_magnitude(top, __shfl_xor_sync(0xffffffffu, top, s));
    if ((threadIdx.x & 31) == 0) warp_top[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) top = max_magnitude(top, warp_top[w]);
    const bool bad = not_finite(top);
    const int e = f8_exponent(top);
    const float inv = bad ? 0.f : exp2_int(-e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        if (r >= rows) break;
        uint2 codes = f8_codes8(v[i], inv);
        if (bad) codes = make_uint2(kF8NanCodes, kF8NanCodes);
        f8_store8(q + (int64_t)r * ldq + c0, cols - c0, codes);
    }
    if (threadIdx.x == 0) {
        scale[(int64_t)blockIdx.y * lds + blockIdx.x] = bad ? __uint_as_float(0x7fc00000u) : exp2_int(e);
        if (bad) report(status, PTQ_ERR_NONFINITE, blockIdx.y * kF8Block);
    }
}

// ------------------------------------------------------------------------------------------------------------
// Product
// ------------------------------------------------------------------------------------------------------------
// K-major operands in rows of 128 bytes, SWIZZLE_128B, 8-row groups 1024 bytes apart (descriptor words as in gram.cuh).
constexpr uint32_t kF8DescHi = (uint32_t)(1024 >> 4) | (1u << 14) | (2u << 29);
constexpr uint32_t kF8DescLo = 1u << 16;
// e4m3 x e4m3 -> float32, M = 128.
__host__ __device__ constexpr uint32_t f8_idesc(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24); }

// The whole warp; one lane issues.
__device__ __forceinline__ void tc_mma_f8(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\t"
                 "mov.b64 da, {%1, %3};\n\t"
                 "mov.b64 db, {%2, %3};\n\t"
                 "setp.ne.b32 p, %5, 0;\n\t"
                 "elect.sync _|e, 0xffffffff;\n\t@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %4, {%6, %6, %6, %6}, p;\n\t}\n"
                 ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(kF8DescHi), "r"(idesc), "r"(accumulate), "r"(0u)
                 : "memory");
}

struct F8Product {
    void* C;
    const float* sa;          // [m][kb], row stride ldsa
    const float* sb;          // [nb][kb], row stride ldsb
    int64_t ldc, ldsa, ldsb;
    int m, n, k, kb;
    int32_t* status;
};

// N consecutive values, in 16-byte pieces where vec says that they begin on 16 bytes.
template <typename T, int N>
__device__ __forceinline__ void store_row(T* p, const float* v, bool vec) {
    if (vec) {
        alignas(16) T t[N];
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = from_f32<T>(v[i]);
#pragma unroll
        for (int i = 0; i < N * (int)sizeof(T) / 16; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = from_f32<T>(v[i]);
    }
}
template <typename T>
__device__ __forceinline__ void store_row16(T* p, const float* v, int n, bool vec) {      // sixteen of which n exist
    if (n >= 16) {
        store_row<T, 16>(p, v, vec);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < n) p[i] = from_f32<T>(v[i]);
    }
}

// Many rows: tiles of 128 rows of A by 256 of B, persistent.  A TMA warp fills four stages of one k block (48 KB); one thread
// issues the four MMAs of a block into one of two TMEM buffers; eight epilogue warps drain the other, one row of the tile and
// 128 columns a thread, and join it to their float32 sums.  128 x 256 x 128 takes the tensor cores 512 clocks; a block takes some
// 1050 here.  8192 x 11008 x 4096: 394 us replayed one after another (1.88 PFLOP/s; 375 for a single launch at a higher clock, and with
// its cast 400 to 480 as a program calls it, by the power limit), of which 60 to 80 go when the epilogue does nothing and another 60 when
// half of B is loaded: 48 KB from L2 for each block of a tile, and the drain of 128 KB of TMEM, hold the tensor cores up in turn.
// (Pairs of SMs on one tile would load a third less; not built.)  A row of C that is no multiple of 16 bytes is stored value by value,
// 32 rows a warp: 2048 x 4095 x 4096 takes 115 us where 2048 x 4096 x 4096 takes 39, 4000 x 1301 x 1024 91 where 4000 x 1304 x 1024 takes 19.
constexpr int kF8TileM = 128, kF8TileN = 256, kF8Stages = 4, kF8Threads = 384;
constexpr int kF8StageBytes = (kF8TileM + kF8TileN) * kF8Block;
constexpr int kF8SmemBytes = 1024 + kF8Stages * kF8StageBytes + 256;
constexpr int kF8GroupM = 16;                 // tiles are taken in groups of this many row blocks, so that a wave shares columns in L2

__device__ __forceinline__ void f8_tile(int tile, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int per = kF8GroupM * tiles_n, g = tile / per, r = tile - g * per;
    const int rows = min(kF8GroupM, tiles_m - g * kF8GroupM);
    tn = r / rows;
    tm = g * kF8GroupM + r - tn * rows;
}

template <typename T>
__global__ void __launch_bounds__(kF8Threads, 1)
f8_product_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, F8Product p, int tiles_m,
                  int tiles_n) {
    chained_wait();
    extern __shared__ unsigned char f8_smem[];
    const uint32_t raw = smem_u32(f8_smem), base = (raw + 1023u) & ~1023u;
    unsigned char* tail = f8_smem + (base - raw) + kF8Stages * kF8StageBytes;
    const uint32_t bar0 = smem_u32(tail);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (kF8Stages + s); };
    auto acc_full = [&](int b) { return bar0 + 8u * (2 * kF8Stages + b); };
    auto acc_empty = [&](int b) { return bar0 + 8u * (2 * kF8Stages + 2 + b); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 8 * (2 * kF8Stages + 4));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, tiles = tiles_m * tiles_n;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kF8Stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), 256); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tc_alloc(smem_u32(tmem_slot), 512u);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);

    // registers: eight epilogue warps with 128 sums each want more than a third of them
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 0) {
            if (lane == 0) {
                int stage = 0, armed[kF8Stages];
                uint32_t phase = 0;
#pragma unroll
                for (int s = 0; s < kF8Stages; ++s) armed[s] = -1;
                bool ok = true;
                for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
                    int tm, tn;
                    f8_tile(tile, tiles_m, tiles_n, tm, tn);
                    for (int b = 0; b < p.kb; ++b) {
                        ok = mbar_wait_bounded(empty_bar(stage), phase ^ 1u, abort_flag);
                        if (!ok) break;
                        const uint32_t dst = base + stage * kF8StageBytes;
                        mbar_arrive_expect_tx(full_bar(stage), kF8StageBytes);
                        armed[stage] = (int)phase;
                        tma_load_2d(dst, &mapA, b * kF8Block, tm * kF8TileM, full_bar(stage));
                        tma_load_2d(dst + kF8TileM * kF8Block, &mapB, b * kF8Block, tn * kF8TileN, full_bar(stage));
                        if (++stage == kF8Stages) { stage = 0; phase ^= 1u; }
                    }
                }
                if (!ok) {
                    for (int s = 0; s < kF8Stages; ++s)
                        if (armed[s] >= 0) drain_copy(full_bar(s), (uint32_t)armed[s]);
                }
            }
        } else if (warp == 1) {
            int stage = 0, buf = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true;
            for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
                for (int b = 0; b < p.kb && ok; ++b) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(acc_empty(buf), acc_phase ^ 1u, abort_flag) &&
                                                     mbar_wait_bounded(full_bar(stage), phase, abort_flag));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t a = kF8DescLo + ((base + stage * kF8StageBytes) >> 4);
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        tc_mma_f8(tmem + buf * kF8TileN, a + 2 * ks, a + 2 * ks + (kF8TileM * kF8Block >> 4), f8_idesc(kF8TileN), ks > 0);
                    tc_commit_elected(empty_bar(stage));
                    tc_commit_elected(acc_full(buf));
                    if (++stage == kF8Stages) { stage = 0; phase ^= 1u; }
                    if (++buf == 2) { buf = 0; acc_phase ^= 1u; }
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        int buf = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        const bool vec = (p.ldc * sizeof(T)) % 16 == 0 && (reinterpret_cast<uintptr_t>(p.C) & 15) == 0;
        const bool sa_vec = p.ldsa % 4 == 0 && (reinterpret_cast<uintptr_t>(p.sa) & 15) == 0;
        for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
            int tm, tn;
            f8_tile(tile, tiles_m, tiles_n, tm, tn);
            const int row = tm * kF8TileM + quarter * 32 + lane, col = tn * kF8TileN + half * kF8Block;
            const bool live = row < p.m && col < p.n;
            const float* sa = p.sa + (int64_t)(live ? row : 0) * p.ldsa;
            const float* sb = p.sb + (int64_t)(col < p.n ? col / kF8Block : 0) * p.ldsb;
            float acc[kF8Block];
#pragma unroll
            for (int c = 0; c < kF8Block; ++c) acc[c] = 0.f;
            // A row's scales come four k blocks at a time and a group ahead: one by one, every lane's load was a sector of its own
            // for each block (8192 x 11008 x 4096 with its cast, replayed: 432 us, 408 so, 400 with two sums an instruction).
            float now[4], ahead[4];
            auto scales = [&](int b) {
                if (sa_vec && b + 4 <= p.kb) {
                    const float4 f = *reinterpret_cast<const float4*>(sa + b);
                    ahead[0] = f.x; ahead[1] = f.y; ahead[2] = f.z; ahead[3] = f.w;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) ahead[j] = b + j < p.kb ? sa[b + j] : 0.f;
                }
            };
            scales(0);
#pragma unroll 1
            for (int b0 = 0; b0 < p.kb && ok; b0 += 4) {
#pragma unroll
                for (int j = 0; j < 4; ++j) now[j] = ahead[j] * (b0 + j < p.kb ? sb[b0 + j] : 0.f);
                if (b0 + 4 < p.kb) scales(b0 + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (b0 + j >= p.kb || !ok) break;
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(acc_full(buf), acc_phase, abort_flag));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + buf * kF8TileN + half * kF8Block;
                    // 16 columns are read while the 16 before them are added
                    uint32_t r[2][16];
                    tc_ld16(taddr, r[0]);
#pragma unroll
                    for (int ch = 0; ch < kF8Block / 16; ++ch) {
                        tc_wait_ld();
                        if (ch + 1 < kF8Block / 16) {
                            tc_ld16(taddr + (ch + 1) * 16, r[(ch + 1) & 1]);
                        } else {
                            tc_fence_before();
                            mbar_arrive(acc_empty(buf));
                        }
#pragma unroll
                        for (int c = 0; c < 16; c += 2) {
                            const float2 sum = fma2(make_float2(__uint_as_float(r[ch & 1][c]), __uint_as_float(r[ch & 1][c + 1])),
                                                    make_float2(now[j], now[j]), make_float2(acc[ch * 16 + c], acc[ch * 16 + c + 1]));
                            acc[ch * 16 + c] = sum.x;
                            acc[ch * 16 + c + 1] = sum.y;
                        }
                    }
                    if (++buf == 2) { buf = 0; acc_phase ^= 1u; }
                }
            }
            if (ok && live) {
                T* out = static_cast<T*>(p.C) + (int64_t)row * p.ldc + col;
#pragma unroll
                for (int c = 0; c < kF8Block; c += 16)
                    if (col + c < p.n) store_row16<T>(out + c, acc + c, p.n - col - c, vec);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tc_dealloc(tmem, 512u);
    if (threadIdx.x == 0 && *abort_flag) report(p.status, PTQ_ERR_TIMEOUT, blockIdx.x);
}

// Few rows: the weights are the 128-row operand of the tensor cores and NT rows of A its columns, so that a single token costs one
// read of the weights and next to nothing else.  KS CTAs of a cluster share a tile's k blocks (one tile of 128 columns alone
// would leave most SMs idle) and join their float32 sums through shared memory, in the order of their ranks.
// One lane holds one column of C: acc[c] += (sa[c][b] sb[b]) d[c], the factors of kF8ScaleBlocks k blocks at a time in shared memory.
constexpr int kF8FewThreads = 192, kF8ScaleBlocks = 16;
template <int NT> struct F8Few {
    static constexpr int stage_bytes = (128 + NT) * kF8Block;
    static constexpr int stages = NT <= 32 ? 5 : 4, bufs = 4;                  // 93 to 106 KB and 64 to 256 columns: two CTAs fit an SM
    static constexpr int columns = bufs * NT;
    static constexpr int scale_bytes = 2 * kF8ScaleBlocks * NT * 4;
    static constexpr int smem_bytes = 1024 + stages * stage_bytes + scale_bytes + 256;
    static_assert(NT * 128 * 4 <= stages * stage_bytes, "the sums go where the stages were");
};

template <typename T, int NT>
__global__ void __launch_bounds__(kF8FewThreads)
f8_product_few_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, F8Product p, int ks_count) {
    using F = F8Few<NT>;
    extern __shared__ unsigned char f8_smem[];
    const uint32_t raw = smem_u32(f8_smem), base = (raw + 1023u) & ~1023u;
    unsigned char* base_ptr = f8_smem + (base - raw);
    float* scales = reinterpret_cast<float*>(base_ptr + F::stages * F::stage_bytes);       // [2][kF8ScaleBlocks][NT]
    unsigned char* tail = base_ptr + F::stages * F::stage_bytes + F::scale_bytes;
    const uint32_t bar0 = smem_u32(tail);
    auto full_bar = [&](int s) { return bar0 + 8u * s; };
    auto empty_bar = [&](int s) { return bar0 + 8u * (F::stages + s); };
    auto acc_full = [&](int b) { return bar0 + 8u * (2 * F::stages + b); };
    auto acc_empty = [&](int b) { return bar0 + 8u * (2 * F::stages + F::bufs + b); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 8 * (2 * F::stages + 2 * F::bufs));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = blockIdx.x, col0 = blockIdx.y * 128, row0 = blockIdx.z * NT;
    const int b0 = (int)((int64_t)p.kb * rank / ks_count), b1 = (int)((int64_t)p.kb * (rank + 1) / ks_count);

    if (threadIdx.x == 0) {
        for (int s = 0; s < F::stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int b = 0; b < F::bufs; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), 128); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tc_alloc(smem_u32(tmem_slot), F::columns);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = (uint32_t)uniform((int)*tmem_slot);
    chained_wait();

    float acc[NT];
    if (warp == 0) {
        if (lane == 0) {
            int stage = 0, armed[F::stages];
            uint32_t phase = 0;
#pragma unroll
            for (int s = 0; s < F::stages; ++s) armed[s] = -1;
            bool ok = true;
            for (int b = b0; b < b1; ++b) {
                ok = mbar_wait_bounded(empty_bar(stage), phase ^ 1u, abort_flag);
                if (!ok) break;
                const uint32_t dst = base + stage * F::stage_bytes;
                mbar_arrive_expect_tx(full_bar(stage), F::stage_bytes);
                armed[stage] = (int)phase;
                tma_load_2d(dst, &mapB, b * kF8Block, col0, full_bar(stage));
                tma_load_2d(dst + 128 * kF8Block, &mapA, b * kF8Block, row0, full_bar(stage));
                if (++stage == F::stages) { stage = 0; phase ^= 1u; }
            }
            if (!ok) {
                for (int s = 0; s < F::stages; ++s)
                    if (armed[s] >= 0) drain_copy(full_bar(s), (uint32_t)armed[s]);
            }
        }
    } else if (warp == 1) {
        int stage = 0, buf = 0;
        uint32_t phase = 0, acc_phase = 0;
        for (int b = b0; b < b1; ++b) {
            if (!__all_sync(0xffffffffu, mbar_wait_bounded(acc_empty(buf), acc_phase ^ 1u, abort_flag) &&
                                             mbar_wait_bounded(full_bar(stage), phase, abort_flag)))
                break;
            tc_fence_after();
            const uint32_t w = kF8DescLo + ((base + stage * F::stage_bytes) >> 4);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                tc_mma_f8(tmem + buf * NT, w + 2 * ks, w + 2 * ks + (128 * kF8Block >> 4), f8_idesc(NT), ks > 0);
            tc_commit_elected(empty_bar(stage));
            tc_commit_elected(acc_full(buf));
            if (++stage == F::stages) { stage = 0; phase ^= 1u; }
            if (++buf == F::bufs) { buf = 0; acc_phase ^= 1u; }
        }
    } else {
        const int quarter = warp & 3, t = threadIdx.x - 64;
        const float* sb = p.sb + (int64_t)blockIdx.y * p.ldsb;
        constexpr int per = NT * kF8ScaleBlocks / 128;
        float ahead[per];
        auto fetch = [&](int b) {                                 // element e: row e / 16 of the tile, k block b + e % 16
#pragma unroll
            for (int i = 0; i < per; ++i) {
                const int e = t + 128 * i, r = row0 + e / kF8ScaleBlocks, bb = b + e % kF8ScaleBlocks;
                ahead[i] = r < p.m && bb < b1 ? p.sa[(int64_t)r * p.ldsa + bb] * sb[bb] : 0.f;
            }
        };
#pragma unroll
        for (int c = 0; c < NT; ++c) acc[c] = 0.f;
        fetch(b0);
        int buf = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        for (int b = b0; b < b1; ++b) {
            const int in = (b - b0) % kF8ScaleBlocks;
            float* now = scales + ((b - b0) / kF8ScaleBlocks & 1) * kF8ScaleBlocks * NT;
            if (in == 0) {
#pragma unroll
                for (int i = 0; i < per; ++i) {
                    const int e = t + 128 * i;
                    now[(e % kF8ScaleBlocks) * NT + e / kF8ScaleBlocks] = ahead[i];
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");    // the four epilogue warps; two buffers, so one barrier is enough
                if (b + kF8ScaleBlocks < b1) fetch(b + kF8ScaleBlocks);
            }
            ok = ok && __all_sync(0xffffffffu, mbar_wait_bounded(acc_full(buf), acc_phase, abort_flag));
            if (!ok) continue;                                    // the barriers above are still met by all four warps
            tc_fence_after();
            const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + buf * NT;
#pragma unroll
            for (int ch = 0; ch < NT / 16; ++ch) {
                uint32_t r[16];
                tc_ld16(taddr + ch * 16, r);
                tc_wait_ld();
#pragma unroll
                for (int c = 0; c < 16; c += 4) {
                    const float4 f = *reinterpret_cast<const float4*>(now + in * NT + ch * 16 + c);
                    acc[ch * 16 + c] = fmaf(f.x, __uint_as_float(r[c]), acc[ch * 16 + c]);
                    acc[ch * 16 + c + 1] = fmaf(f.y, __uint_as_float(r[c + 1]), acc[ch * 16 + c + 1]);
                    acc[ch * 16 + c + 2] = fmaf(f.z, __uint_as_float(r[c + 2]), acc[ch * 16 + c + 2]);
                    acc[ch * 16 + c + 3] = fmaf(f.w, __uint_as_float(r[c + 3]), acc[ch * 16 + c + 3]);
                }
            }
            tc_fence_before();
            mbar_arrive(acc_empty(buf));
            if (++buf == F::bufs) { buf = 0; acc_phase ^= 1u; }
        }
    }
    tc_fence_before();
    __syncthreads();                       // every copy has been multiplied and every product read: the stages are free
    tc_fence_after();
    if (warp == 1) tc_dealloc(tmem, F::columns);
    float* sums = reinterpret_cast<float*>(base_ptr);                          // [NT][128]
    const int lane_col = (warp & 3) * 32 + lane, col = col0 + lane_col;
    T* out = static_cast<T*>(p.C) + col;
    if (ks_count > 1) {
        if (warp >= 2) {
#pragma unroll
            for (int c = 0; c < NT; ++c) sums[c * 128 + lane_col] = acc[c];
        }
        cluster_barrier();
        if (warp >= 2 && col < p.n) {
            const uint32_t at = smem_u32(sums + lane_col);
            for (int c = NT * rank / ks_count; c < NT * (rank + 1) / ks_count && row0 + c < p.m; ++c) {
                float s = 0.f;
                for (int r = 0; r < ks_count; ++r) s += load_cluster_f32(at + c * 512u, r);
                out[(int64_t)(row0 + c) * p.ldc] = from_f32<T>(s);
            }
        }
        cluster_barrier();                 // no CTA leaves while another reads its sums
    } else if (warp >= 2 && col < p.n) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
            if (row0 + c < p.m) out[(int64_t)(row0 + c) * p.ldc] = from_f32<T>(acc[c]);
    }
    if (threadIdx.x == 0 && *abort_flag) report(p.status, PTQ_ERR_TIMEOUT, blockIdx.y);
}

inline int f8_map(CUtensorMap* m, const uint8_t* q, int rows, int cols, int64_t ld, int box_rows) {
    EncodeTiledFn enc = get_encode_tiled();
    if (!enc) return PTQ_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kF8Block, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1u, 1u};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(q), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? PTQ_OK : PTQ_ERR_CUDA;
}

}  // namespace ptq
