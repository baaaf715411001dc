// Matrix product with bias, activation and residual in its epilogue, Y = f(X W^T + b) + R, and the products
// of its backward pass, dX = dZ W and dW = dZ^T X with dZ = dY f'(Z), on the tensor cores (bf16 x bf16 ->
// fp32 in tensor memory).
//
// All three are D(r, c) = sum_k P(r, k) Q(c, k); they differ in which index of P and Q is contiguous:
//     Y:  P = X (k contiguous)      Q = W (k contiguous)       k = input feature
//     dX: P = dZ (k contiguous)     Q = W^T (c contiguous)     k = output feature
//     dW: P = dZ^T (r contiguous)   Q = X^T (c contiguous)     k = token
// The tensor core takes either order from shared memory, so nothing is transposed; the order is a field of
// the instruction descriptor and a choice of boxes for the tensor copies.
//
// Two kernels.  pair: 256 x 256 tiles on CTA pairs, for many rows.  slim: few tokens, where reading W once is
// the work: W's rows are the tensor core's 128 rows and the tokens its columns, so that no row of the
// instruction is wasted, and the contraction is split over the CTAs of a cluster, which join their partial
// sums through distributed shared memory in a fixed order.
//
// Precision: the tensor core's fp32 accumulator loses what a sum rounded to nearest would not, always towards zero, and
// the more the longer the sum: 1.0e-6 of the result over 1000 terms, 4.4e-6 over 4096, 9.1e-6 over 8192.  Where the result
// is fp32, an accumulator therefore takes a few blocks of k and is then folded: the epilogue's warps add it to a sum in
// their registers, rounded to nearest, while the tensor cores fill the other one.  4.6e-7 to 6.5e-7 at any length, for 11 %
// of the time (4096 x 4096 x 4096, fp32: 108 us, 97 in one accumulator).  Results in bf16 are rounded far above either.
//
// Every wait on an mbarrier is bounded by a clock budget; on expiry the error word is set and the CTA drains.
#include <cuda.h>
#include <cuda_bf16.h>

#include "bf16_mma.cuh"
#include "common.cuh"
#include "waits.cuh"

namespace dastac {
namespace {

constexpr int kBlockK = 64;
constexpr int kFoldBlocks = 8;
// Blocks of k that an accumulator takes, with `left` of `all` to go.  The first one of a long contraction takes twice as many:
// the tensor cores work on it while the epilogue of the tile before still holds the other (4096 x 4096 x 4096, fp32: 108 us,
// 113 with equal parts).
__device__ __forceinline__ int fold_blocks(int left, int all) {
    const int most = left == all && all >= 4 * kFoldBlocks ? 2 * kFoldBlocks : kFoldBlocks;
    return left < most ? left : most;
}
enum ErrCode : int32_t { kErrFull = 0x4c01, kErrEmpty = 0x4c03, kErrTmemFull = 0x4c04, kErrTmemEmpty = 0x4c05 };

// ---- activations -------------------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid_of(float z) {
    // exp(-z) is infinite below -88, and its reciprocal the 0 that is due; the reciprocal takes that and NaN as they are
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + __expf(-z)));
    return r;
}
// Phi(z) = (1 + erf(z / sqrt 2)) / 2 by the rational form of Abramowitz and Stegun 7.1.26 (absolute error of erf
// below 1.5e-7) and, from the same exponential, the density of the normal distribution.
__device__ __forceinline__ float normal_cdf(float z, float& density) {
    const float x = fabsf(z) * 0.70710678118654752f;
    const float t = __fdividef(1.f, fmaf(0.3275911f, x, 1.f));
    const float e = __expf(-x * x);
    float q = fmaf(1.061405429f, t, -1.453152027f);
    q = fmaf(q, t, 1.421413741f);
    q = fmaf(q, t, -0.284496736f);
    q = fmaf(q, t, 0.254829592f);
    const float tail = 0.5f * q * t * e;   // Phi(-|z|)
    density = 0.39894228040143268f * e;
    return z > 0.f ? 1.f - tail : tail;
}
template <int ACT>
__device__ __forceinline__ float act_of(float z) {
    if (ACT == DASTAC_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    if (ACT == DASTAC_ACT_SIGMOID) return sigmoid_of(z);
    if (ACT == DASTAC_ACT_SILU) return z * sigmoid_of(z);
    if (ACT == DASTAC_ACT_GELU) {
        float density;
        return z * normal_cdf(z, density);
    }
    return z;
}
template <int ACT>
__device__ __forceinline__ float slope_of(float z) {
    if (ACT == DASTAC_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    if (ACT == DASTAC_ACT_SIGMOID) return sigmoid_of(z) * sigmoid_of(-z);
    if (ACT == DASTAC_ACT_SILU) return sigmoid_of(z) * (1.f + z * sigmoid_of(-z));
    if (ACT == DASTAC_ACT_GELU) {
        float density;
        const float p = normal_cdf(z, density);
        return fmaf(z, density, p);
    }
    return 1.f;
}

// ---- one product and what happens to its result --------------------------------------------------------
struct Problem {
    int32_t a_mn, b_mn;                      // the operand's row index is the contiguous one
    int32_t k_blocks, row_blocks, col_blocks;  // blocks of 64, 256 and 256
    int32_t k_wrap;   // from this k on Q is read from its beginning again (P is two parts behind one another); a_mn and b_mn only
    int32_t act, out_dtype, accumulate;
    int32_t fold;     // pairs: accumulators are added to sums in registers every few blocks of k
    int32_t even, quad, whole, wide;   // out, z and residual take 2 columns, 4 columns, 16 bytes, 32 bytes in an aligned access
    int64_t rows, cols;
    void* out;
    int64_t ld;
    const float* bias;
    const void* residual;
    int64_t ldr;
    __nv_bfloat16* z;
    int64_t ldz;
};

// ---- pair: 256 x 256 tiles on CTA pairs ----------------------------------------------------------------
// CTA r of a pair stages rows 128 r .. of the tile's P block and columns 128 r .. of its Q block (16 KiB
// each per 64 of k), and holds the 128 x 256 accumulator of its own rows, double buffered in tensor memory:
// eight epilogue warps drain one buffer (warp w: lanes 32 (w mod 4) .., column half w / 4) while the MMAs of
// the next tile fill the other.  CTA 0 issues the MMAs; its barriers count both CTAs' copies.
//
// The epilogue takes 32 x 32 values a warp at a time; a thread has a row of the accumulator in its registers.
// DIRECT: rows whose pieces of 16 bytes are aligned go from there to memory, a whole sector a store (or half of one), which
// leaves all of shared memory to the stages: the main loop is bound by the bytes in flight (a stage is loaded,
// waits, is multiplied and is freed in about 2 us, so seven stages of 64 of k bring 0.3 us a stage, what the tensor
// cores take).  Otherwise a warp turns its block in shared memory, at the price of a stage, and half a warp
// stores a row, two columns a thread: whole segments for any pitch.
//
// Measured: 8192 rows, 4096 by 8192, GELU with z kept: 371 us, 1480 TFLOP/s, the tensor pipe active for 94 % of
// the cycles; bound by the tensor cores at the clock that the power limit leaves.  1017 rows, 1000 by 2501, rows not
// aligned, fp32 result: 20 us, 40 tiles on 74 pairs, each a launch, a pipeline to fill and an epilogue in a row.
template <bool DIRECT>
constexpr int kStagesOf = DIRECT ? 7 : 6;
constexpr int kOperandBytes = 128 * kBlockK * 2;
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kEpiWarps = 8;
constexpr int kWarpTma = kEpiWarps, kWarpMma = kEpiWarps + 1;
constexpr int kPairThreads = 32 * (kEpiWarps + 2);
constexpr int kEpiPitch = 33;
constexpr int kEpiBytes = 32 * kEpiPitch * 4;
template <bool DIRECT>
constexpr size_t kPairSmem = (size_t)kStagesOf<DIRECT> * kStageBytes + (DIRECT ? 0 : kEpiWarps * kEpiBytes) + 256 + 1024;
static_assert(kPairSmem<true> <= 232448 && kPairSmem<false> <= 232448, "shared memory of a CTA");
constexpr int kTmemCols = 512;

// A look at a stage that does not wait: of the next one, while this one's MMAs are issued.
__device__ __forceinline__ bool peek(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The MMA and its commit by one elected lane of a converged warp: descriptors stay in uniform registers, which a branch
// on the lane would take away.
__device__ __forceinline__ void umma_elected_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void commit_elected_pair(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
        ::"r"(bar), "h"((uint16_t)3)
        : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) { asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory"); }

struct True {
    static constexpr bool value = true;
};
struct False {
    static constexpr bool value = false;
};

struct PairParams {
    Problem q[2];
    int64_t tiles0, tiles;  // of the first problem, of both
    int32_t* err_word;
};

// fp32 accumulator, bf16 operands; bits 15 and 16: the row index of A / B is the contiguous one
__device__ __forceinline__ uint32_t instruction(int m, int n, int a_mn, int b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(m >> 4) << 24);
}
// Operand descriptor of a staged block of 64 of k, and what the next 16 of k add to it: k contiguous (rows of 128
// bytes, 8 rows 1024 bytes apart) or rows contiguous (64 x 64 sub-blocks of 8 KiB).
__device__ __forceinline__ uint64_t operand(uint32_t addr, bool mn) { return smem_desc(addr, mn ? 64 * 128 : 16, 1024); }
constexpr uint64_t kNextK = 32 >> 4, kNextMn = 2048 >> 4;

// A wait as the one thread of a role needs it: a stage is mostly ready, and the loop around it is bound by the
// latency of its instructions, so the bounded wait stays out of line.
__device__ __noinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* err_word, int32_t code) {
    return mbar_wait(bar, parity, abort_flag, err_word, code);
}
__device__ __forceinline__ bool wait_stage(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* err_word, int32_t code) {
    return mbar_test(bar, parity) || wait_slow(bar, parity, abort_flag, err_word, code);
}
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Eight 32-bit words, aligned to 32 bytes.
__device__ __forceinline__ void store8(void* p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                 "r"(w[6]), "r"(w[7])
                 : "memory");
}
__device__ __forceinline__ void load8(const void* p, uint32_t (&w)[8]) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
}
// A thread's 32 values of a row, n of them inside the matrix, from / to memory aligned to 16 bytes (`wide`: to 32).
template <typename T>
__device__ __forceinline__ void add_row(const T* p, float (&v)[32], int n, bool wide) {
    constexpr int kPiece = 32 / sizeof(T);
#pragma unroll
    for (int k = 0; k < 32; k += kPiece) {
        if (k + kPiece <= n) {
            uint32_t w[8];
            if (wide) {
                load8(p + k, w);
            } else {
                const uint4 lo = *(const uint4*)(p + k), hi = *(const uint4*)(p + k + kPiece / 2);
                w[0] = lo.x, w[1] = lo.y, w[2] = lo.z, w[3] = lo.w, w[4] = hi.x, w[5] = hi.y, w[6] = hi.z, w[7] = hi.w;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (sizeof(T) == 4) {
                    v[k + e] += __uint_as_float(w[e]);
                } else {
                    v[k + 2 * e] += __uint_as_float(w[e] << 16);
                    v[k + 2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u);
                }
            }
        } else {
#pragma unroll
            for (int e = k; e < k + kPiece; ++e)
                if (e < n) v[e] += (float)p[e];
        }
    }
}
template <typename T>
__device__ __forceinline__ void store_row(T* p, const float (&v)[32], int n, bool wide) {
    constexpr int kPiece = 32 / sizeof(T);
#pragma unroll
    for (int k = 0; k < 32; k += kPiece) {
        if (k + kPiece <= n) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(v[k + e]);
                else w[e] = bf16_pair(v[k + 2 * e], v[k + 2 * e + 1]);
            }
            if (wide) {
                store8(p + k, w);
            } else {
                *(uint4*)(p + k) = make_uint4(w[0], w[1], w[2], w[3]);
                *(uint4*)(p + k + kPiece / 2) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        } else {
#pragma unroll
            for (int e = k; e < k + kPiece; ++e)
                if (e < n) p[e] = (T)v[e];
        }
    }
}

// 32 x 32 values out of shared memory (pitch 33) into a matrix of any alignment, `add` to be added first: a lane a
// column, or half a warp a row with two columns a lane where pairs are aligned (`even`).
template <typename T>
__device__ __forceinline__ void store_block(const float* stage, T* out, int64_t ld, const T* add, int64_t lda, int rows, int n, bool even, int lane) {
    if (even && n % 2 == 0) {
        const int c = 2 * (lane & 15);
        if (c >= n) return;
#pragma unroll 4
        for (int i = lane >> 4; i < rows; i += 2) {
            float x = stage[i * kEpiPitch + c], y = stage[i * kEpiPitch + c + 1];
            if constexpr (sizeof(T) == 4) {
                if (add) {
                    const float2 w = *(const float2*)(add + i * lda + c);
                    x += w.x;
                    y += w.y;
                }
                *(float2*)(out + i * ld + c) = make_float2(x, y);
            } else {
                if (add) {
                    const float2 w = __bfloat1622float2(*(const __nv_bfloat162*)(add + i * lda + c));
                    x += w.x;
                    y += w.y;
                }
                *(__nv_bfloat162*)(out + i * ld + c) = __floats2bfloat162_rn(x, y);
            }
        }
    } else {
        if (lane >= n) return;
        T* o = out + lane;
        if (add) {
            const T* a = add + lane;
#pragma unroll 8
            for (int i = 0; i < rows; ++i) o[i * ld] = (T)(stage[i * kEpiPitch + lane] + (float)a[i * lda]);
        } else {
#pragma unroll 8
            for (int i = 0; i < rows; ++i) o[i * ld] = (T)stage[i * kEpiPitch + lane];
        }
    }
}

// A warp's 32 rows x 128 columns of a tile.
template <int ACT, bool DIRECT>
__device__ __forceinline__ void pair_epilogue(const Problem& q, uint32_t taddr, float* stage, int64_t row0, int64_t col0, int lane) {
    const int rows = (int)min((int64_t)32, q.rows - row0);
    const void* const add = q.accumulate ? q.out : q.residual;
    const int64_t lda = q.accumulate ? q.ld : q.ldr;
#pragma unroll 1
    for (int cc = 0; cc < 4; ++cc) {
        const int64_t c0 = col0 + 32 * cc;
        if (c0 >= q.cols) break;   // the same for the whole warp
        const int n = (int)min((int64_t)32, q.cols - c0);
        float v[32];
        {
            uint32_t w[32];
            tmem_ld32(taddr + 32 * cc, w);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = q.k_blocks ? __uint_as_float(w[j]) : 0.f;
        }
        if (q.bias) {   // the same word for all lanes
            if (n == 32 && ((uintptr_t)q.bias & 15) == 0) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float4 b = __ldg((const float4*)(q.bias + c0) + k);
                    v[4 * k] += b.x;
                    v[4 * k + 1] += b.y;
                    v[4 * k + 2] += b.z;
                    v[4 * k + 3] += b.w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (j < n) v[j] += __ldg(q.bias + c0 + j);
            }
        }
        if constexpr (DIRECT) {
            const int64_t r = row0 + lane;
            if (lane < rows) {
                if (q.z) store_row(q.z + r * q.ldz + c0, v, n, q.wide);
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = act_of<ACT>(v[j]);
                if (q.out_dtype == DASTAC_F32) {
                    if (add) add_row((const float*)add + r * lda + c0, v, n, q.wide);
                    store_row((float*)q.out + r * q.ld + c0, v, n, q.wide);
                } else {
                    if (add) add_row((const __nv_bfloat16*)add + r * lda + c0, v, n, q.wide);
                    store_row((__nv_bfloat16*)q.out + r * q.ld + c0, v, n, q.wide);
                }
            }
        } else {
            __syncwarp();
            if (q.z) {
#pragma unroll
                for (int j = 0; j < 32; ++j) stage[lane * kEpiPitch + j] = v[j];
                __syncwarp();
                store_block<__nv_bfloat16>(stage, q.z + row0 * q.ldz + c0, q.ldz, nullptr, 0, rows, n, q.even, lane);
                __syncwarp();
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) stage[lane * kEpiPitch + j] = act_of<ACT>(v[j]);
            __syncwarp();
            if (q.out_dtype == DASTAC_F32)
                store_block<float>(stage, (float*)q.out + row0 * q.ld + c0, q.ld, add ? (const float*)add + row0 * lda + c0 : nullptr, lda, rows, n,
                                   q.even, lane);
            else
                store_block<__nv_bfloat16>(stage, (__nv_bfloat16*)q.out + row0 * q.ld + c0, q.ld,
                                           add ? (const __nv_bfloat16*)add + row0 * lda + c0 : nullptr, lda, rows, n, q.even, lane);
        }
    }
}

template <bool DIRECT, bool FOLD>   // FOLD: some problem asks for it
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap b0,
                   const __grid_constant__ CUtensorMap a1, const __grid_constant__ CUtensorMap b1, const __grid_constant__ PairParams p) {
    constexpr int kStages = kStagesOf<DIRECT>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* epi = smem + (size_t)kStages * kStageBytes;
    uint64_t* bars = (uint64_t*)(epi + (DIRECT ? 0 : kEpiWarps * kEpiBytes));
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (kStages + s); };
    auto tmem_full = [&](int a) { return bar0 + 8u * (2 * kStages + a); };
    auto tmem_empty = [&](int a) { return bar0 + 8u * (2 * kStages + 2 + a); };
    const uint32_t drain_bar = bar0 + 8u * (2 * kStages + 4);
    uint32_t* tmem_slot = (uint32_t*)(bars + 2 * kStages + 5);
    volatile int* abort_flag = (volatile int*)(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem_base = smem_u32(smem);
    const uint32_t rank = cluster_ctarank();

    if (warp == kWarpTma && lane == 0) {
        prefetch_map(&a0);
        prefetch_map(&b0);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tmem_full(a), 1);
            mbar_init(tmem_empty(a), 2 * kEpiWarps);
        }
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kWarpMma) {
        tmem_alloc_pair(smem_u32(tmem_slot), kTmemCols);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    // Tile t: the first problem's tiles (the longer contraction) before the second's; within a problem
    // bands of eight row blocks, column by column, so that the tiles in flight share operands in L2.  Tiles
    // are dealt to the clusters in boustrophedon order, which evens out the two lengths.
    const int64_t G = gridDim.x >> 1, cid = blockIdx.x >> 1;
    const uint32_t rounds = (uint32_t)((p.tiles + G - 1) / G);
    auto tile_of = [&](uint32_t n) -> int64_t { return (int64_t)n * G + ((n & 1) ? (G - 1 - cid) : cid); };
    auto locate = [&](int64_t t, int& which, int& R, int& C) {
        which = t >= p.tiles0;
        if (which) t -= p.tiles0;
        const Problem& q = p.q[which];
        const int64_t band = t / (8LL * q.col_blocks);
        const int height = min(8, q.row_blocks - (int)band * 8);
        const int in_band = (int)(t - band * 8 * q.col_blocks);
        R = (int)band * 8 + in_band % height;
        C = in_band / height;
    };

    if (warp == kWarpTma) {
        if (lane == 0) {
            const uint32_t full0 = map_to_cta(full(0), 0);
            Turn turn{0, 1};   // a fresh barrier's phase before the first counts as complete
            bool ok = true;
            // the copies of a tile, for each order of the operands
            auto copy_tile = [&](const CUtensorMap* ma, const CUtensorMap* mb, int ra, int rb, int k_blocks, int k_wrap, auto a_mn, auto b_mn) {
                for (int k = 0; k < k_blocks * kBlockK; k += kBlockK, turn.next(kStages)) {
                    if (!wait_stage(empty(turn.s), turn.parity, abort_flag, p.err_word, kErrEmpty)) return false;
                    const uint32_t dst = smem_base + turn.s * kStageBytes, bar = full0 + 8u * turn.s;
                    if (rank == 0) mbar_arrive_expect_tx(full(turn.s), 2 * kStageBytes);
                    if constexpr (a_mn.value) {
                        tma_load_2d_pair(dst, ma, ra, k, bar);
                        tma_load_2d_pair(dst + 8192, ma, ra + 64, k, bar);
                    } else {
                        tma_load_2d_pair(dst, ma, k, ra, bar);
                    }
                    if constexpr (b_mn.value) {
                        const int kq = a_mn.value && k >= k_wrap ? k - k_wrap : k;
                        tma_load_2d_pair(dst + kOperandBytes, mb, rb, kq, bar);
                        tma_load_2d_pair(dst + kOperandBytes + 8192, mb, rb + 64, kq, bar);
                    } else {
                        tma_load_2d_pair(dst + kOperandBytes, mb, k, rb, bar);
                    }
                }
                return true;
            };
            for (uint32_t n = 0; n < rounds && ok; ++n) {
                const int64_t t = tile_of(n);
                if (t >= p.tiles) continue;
                int which, R, C;
                locate(t, which, R, C);
                const Problem& q = p.q[which];
                const CUtensorMap* ma = which ? &a1 : &a0;
                const CUtensorMap* mb = which ? &b1 : &b0;
                const int ra = R * 256 + (int)rank * 128, rb = C * 256 + (int)rank * 128;
                if (q.a_mn) ok = copy_tile(ma, mb, ra, rb, q.k_blocks, q.k_wrap, True{}, True{});
                else if (q.b_mn) ok = copy_tile(ma, mb, ra, rb, q.k_blocks, q.k_wrap, False{}, True{});
                else ok = copy_tile(ma, mb, ra, rb, q.k_blocks, q.k_wrap, False{}, False{});
            }
            if (!ok) {   // give copies in flight time to land before shared memory is released
                const long long t0 = clock64();
                while (clock64() - t0 < 2000000) {
                }
            }
        }
    } else if (warp == kWarpMma) {
        if (rank == 0) {
            Turn turn{0, 0};
            uint32_t pass_n = 0;
            bool ok = true;
            const uint64_t a_k = operand(smem_base, false), a_m = operand(smem_base, true);
            auto multiply_tile = [&](uint32_t d_tmem, uint64_t a, uint64_t b, uint64_t a_next, uint64_t b_next, uint32_t idesc, int k_blocks) {
                bool ready = false;
                for (int kb = 0; kb < k_blocks; ++kb) {
                    if (!__all_sync(~0u, ready || wait_stage(full(turn.s), turn.parity, abort_flag, p.err_word, kErrFull))) return false;
                    tc_fence_after();
                    const uint64_t at = (uint64_t)(turn.s * (kStageBytes >> 4));
                    const uint32_t release = empty(turn.s);
                    turn.next(kStages);
                    ready = kb + 1 < k_blocks && peek(full(turn.s), turn.parity);
#pragma unroll
                    for (int k16 = 0; k16 < kBlockK / 16; ++k16)
                        umma_elected_pair(d_tmem, a + at + k16 * a_next, b + at + k16 * b_next, idesc, (kb > 0 || k16 > 0) ? 1u : 0u);
                    commit_elected_pair(release);
                }
                return true;
            };
            for (uint32_t n = 0; n < rounds && ok; ++n) {
                const int64_t t = tile_of(n);
                if (t >= p.tiles) continue;
                int which, R, C;
                locate(t, which, R, C);
                const Problem& q = p.q[which];
                const uint64_t b0d = (q.b_mn ? a_m : a_k) + (kOperandBytes >> 4);
                int left = q.k_blocks;
                do {   // an accumulator at a time: all of the contraction, or a few blocks of it
                    const int acc = pass_n & 1, blocks = FOLD && q.fold ? fold_blocks(left, q.k_blocks) : left;
                    const uint32_t use = pass_n >> 1;
                    if (use >= 1 && !__all_sync(~0u, wait_stage(tmem_empty(acc), (use - 1) & 1, abort_flag, p.err_word, kErrTmemEmpty))) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    ok = multiply_tile(tmem_base + acc * 256, q.a_mn ? a_m : a_k, b0d, q.a_mn ? kNextMn : kNextK, q.b_mn ? kNextMn : kNextK,
                                       instruction(256, 256, q.a_mn, q.b_mn), blocks);
                    if (ok) commit_elected_pair(tmem_full(acc));
                    ++pass_n;
                    left -= blocks;
                } while (ok && left > 0);
            }
            if (!ok) {
                commit_elected_pair(drain_bar);
                const long long t0 = clock64();
                while (!mbar_test(drain_bar, 0) && clock64() - t0 < kWaitBudget) {
                }
            }
        }
    } else {
        const uint32_t empty0 = map_to_cta(tmem_empty(0), 0);
        const int quarter = warp & 3, half = warp >> 2;
        float* const stage = (float*)(epi + warp * kEpiBytes);
        uint32_t pass_n = 0;
        bool ok = true;
        for (uint32_t n = 0; n < rounds && ok; ++n) {
            const int64_t t = tile_of(n);
            if (t >= p.tiles) continue;
            int which, R, C;
            locate(t, which, R, C);
            const Problem& q = p.q[which];
            uint32_t taddr;
            auto wait_accumulator = [&]() {
                const int acc = pass_n & 1;
                if (!mbar_wait_warp(tmem_full(acc), (pass_n >> 1) & 1, abort_flag, p.err_word, kErrTmemFull, lane)) return false;
                tc_fence_after();
                taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + acc * 256 + half * 128;
                return true;
            };
            auto free_accumulator = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(empty0 + 8u * (pass_n & 1));
                ++pass_n;
            };
            ok = wait_accumulator();
            if (!ok) break;
            const int64_t row0 = (int64_t)R * 256 + rank * 128 + quarter * 32, col0 = (int64_t)C * 256 + half * 128;
            if (FOLD && q.fold) {   // the accumulators in turn, their sum back into the last one
                float sum[8][16];
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c][j] = 0.f;
                int left = q.k_blocks;
                while (true) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        uint32_t w[16];
                        tmem_ld16(taddr + 16 * c, w);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[c][j] += __uint_as_float(w[j]);
                    }
                    left -= fold_blocks(left, q.k_blocks);
                    if (left == 0) break;
                    free_accumulator();
                    ok = wait_accumulator();
                    if (!ok) break;
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(sum[c][j]);
                    tmem_st16(taddr + 16 * c, w);
                }
                tmem_st_wait();
            }
            if (row0 < q.rows) switch (q.act) {
                case DASTAC_ACT_RELU: pair_epilogue<DASTAC_ACT_RELU, DIRECT>(q, taddr, stage, row0, col0, lane); break;
                case DASTAC_ACT_SIGMOID: pair_epilogue<DASTAC_ACT_SIGMOID, DIRECT>(q, taddr, stage, row0, col0, lane); break;
                case DASTAC_ACT_SILU: pair_epilogue<DASTAC_ACT_SILU, DIRECT>(q, taddr, stage, row0, col0, lane); break;
                case DASTAC_ACT_GELU: pair_epilogue<DASTAC_ACT_GELU, DIRECT>(q, taddr, stage, row0, col0, lane); break;
                default: pair_epilogue<DASTAC_ACT_NONE, DIRECT>(q, taddr, stage, row0, col0, lane); break;
            }
            free_accumulator();
        }
    }
    // Neither CTA may leave, or give back tensor memory, while its peer can still touch it.
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == kWarpMma) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, kTmemCols);
    }
}

// ---- slim: few tokens, and products with too few tiles for the pairs ---------------------------------------
// D(n, m) with 128 rows of W a CTA and `tokens` columns (16, 32, 64 or 128); the CTAs of a cluster share one
// tile and take equal parts of the contraction.  The partial sums meet in the cluster's shared memory: rank
// s of S sums columns s, s + S, ... over the ranks in order.  With few tokens memory is what bounds this kernel,
// so a stage ring of up to 200 KB keeps that much of W in flight per SM.
//
// Measured: 32 rows, 16384 by 4096: 26 us, 5.2 TB/s, bound by memory; 1 row, 4096 by 4096: 9.3 us, 3.6 TB/s,
// of which 5.1 us are the weights at the rate of a copy and the rest is the launch, the first bytes' latency, the
// join and the epilogue.  256 and 512 rows, 4096 by 4096: 17 and 26 us, a whole tile through one CTA with nothing behind it.
constexpr int kSlimEpi = 8, kSlimTma = 8, kSlimMma = 9;   // warps
constexpr int kSlimThreads = 32 * (kSlimEpi + 2);
constexpr size_t kSlimMax = 232448 - 2048;
constexpr size_t kSlimLeast = 40960;

struct SlimParams {
    Problem q;            // rows = tokens, cols = output features, as for the pair kernel
    int32_t tokens;       // columns of the instruction
    int32_t stages;
    int32_t* err_word;
};

__device__ __forceinline__ void tmem_alloc_one(uint32_t slot, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_one(uint32_t taddr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
__device__ __forceinline__ void umma_elected_one(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void commit_elected_one(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar)
        : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// The tokens of this rank, a warp each: a lane sums four neighbouring columns over the ranks in order and finishes them.
// part[source][token of this rank][128 columns]
template <int ACT>
__device__ __forceinline__ void slim_finish(const Problem& q, const float* part, int tokens, int ranks, int rank, int64_t m0, int64_t n0, int warp,
                                            int lane) {
    const int mine = (tokens - rank + ranks - 1) / ranks, most = (tokens + ranks - 1) / ranks;
    const int64_t n = n0 + 4 * lane;
    const int cols = (int)max((int64_t)0, min((int64_t)4, q.cols - n));
    if (cols == 0) return;
    const bool whole = cols == 4 && q.quad;
    float bias[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) bias[j] = q.bias && j < cols ? __ldg(q.bias + n + j) : 0.f;
    const void* const add = q.accumulate ? q.out : q.residual;
    const int64_t lda = q.accumulate ? q.ld : q.ldr;
    const int live = (int)min((int64_t)mine, (q.rows - m0 - rank + ranks - 1) / ranks);
#pragma unroll 2
    for (int i = warp; i < live; i += kSlimEpi) {
        const int64_t m = m0 + rank + (int64_t)i * ranks;
        float v[4] = {0.f, 0.f, 0.f, 0.f}, r[4] = {0.f, 0.f, 0.f, 0.f};
        if (add) {
            if (q.out_dtype == DASTAC_F32) {
                const float* p = (const float*)add + m * lda + n;
                if (whole) {
                    const float4 w = *(const float4*)p;
                    r[0] = w.x, r[1] = w.y, r[2] = w.z, r[3] = w.w;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < cols) r[j] = p[j];
                }
            } else {
                const __nv_bfloat16* p = (const __nv_bfloat16*)add + m * lda + n;
                if (whole) {
                    const uint2 w = *(const uint2*)p;
                    r[0] = __uint_as_float(w.x << 16), r[1] = __uint_as_float(w.x & 0xffff0000u);
                    r[2] = __uint_as_float(w.y << 16), r[3] = __uint_as_float(w.y & 0xffff0000u);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (j < cols) r[j] = __bfloat162float(p[j]);
                }
            }
        }
        if (q.k_blocks)
            for (int s = 0; s < ranks; ++s) {
                const float4 w = *(const float4*)(part + (s * most + i) * 128 + 4 * lane);
                v[0] += w.x, v[1] += w.y, v[2] += w.z, v[3] += w.w;
            }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] += bias[j];
        if (q.z) {
            __nv_bfloat16* p = q.z + m * q.ldz + n;
            if (whole) {
                *(uint2*)p = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < cols) p[j] = __float2bfloat16_rn(v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = act_of<ACT>(v[j]) + r[j];
        if (q.out_dtype == DASTAC_F32) {
            float* p = (float*)q.out + m * q.ld + n;
            if (whole) {
                *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < cols) p[j] = v[j];
            }
        } else {
            __nv_bfloat16* p = (__nv_bfloat16*)q.out + m * q.ld + n;
            if (whole) {
                *(uint2*)p = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < cols) p[j] = __float2bfloat16_rn(v[j]);
            }
        }
    }
}

// How a CTA's sum is kept: in one accumulator; in two that take the blocks of k in turn and are added at the end (fp32
// results, up to 2 kFoldBlocks blocks of k); folded (fp32 results, more blocks).  1 x 4096 x 4096, 16 blocks a CTA: 8.3 us in two
// accumulators, 8.9 folded; 128 x 19000 x 8192, 128 blocks: 87.8 us folded, 85.4 in two with three times the error.
enum Sums { kOneSum, kTwoSums, kFolded };
template <Sums SUMS>
__global__ void __launch_bounds__(kSlimThreads, 1)
linear_slim_kernel(const __grid_constant__ CUtensorMap mw, const __grid_constant__ CUtensorMap mx, const __grid_constant__ SlimParams p) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int stages = p.stages, tokens = p.tokens;
    const int x_bytes = tokens * kBlockK * 2, stage_bytes = kOperandBytes + x_bytes;
    uint32_t ranks;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const uint32_t rank = cluster_ctarank();
    float* part = (float*)(smem + (size_t)stages * stage_bytes);
    const int most = (tokens + (int)ranks - 1) / (int)ranks;
    uint64_t* bars = (uint64_t*)(part + (size_t)ranks * most * 128);
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (stages + s); };
    auto tmem_full = [&](uint32_t a) { return bar0 + 8u * (2 * stages + a); };
    auto tmem_empty = [&](uint32_t a) { return bar0 + 8u * (2 * stages + 2 + a); };
    uint32_t* tmem_slot = (uint32_t*)(bars + 2 * stages + 4);
    volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t smem_base = smem_u32(smem);
    const int each = tokens < 32 ? 32 : tokens;   // columns of an accumulator
    const uint32_t tmem_cols = SUMS == kOneSum ? each : 2 * each;

    if (warp == kSlimTma && lane == 0) {
        prefetch_map(&mw);
        prefetch_map(&mx);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tmem_full(a), 1);
            mbar_init(tmem_empty(a), kSlimEpi);
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kSlimMma) tmem_alloc_one(smem_u32(tmem_slot), tmem_cols);
    tc_fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    const Problem& q = p.q;
    const int64_t n0 = (int64_t)(blockIdx.x / ranks) * 128, m0 = (int64_t)blockIdx.y * tokens;
    const int k_begin = (int)((int64_t)q.k_blocks * rank / ranks), k_end = (int)((int64_t)q.k_blocks * (rank + 1) / ranks);

    if (warp == kSlimTma) {
        if (lane == 0) {
            Turn turn{0, 1};
            bool fine = true;
            const int wide = q.b_mn;
            for (int k = k_begin * kBlockK; k < k_end * kBlockK; k += kBlockK, turn.next(stages)) {
                const uint32_t bar = full(turn.s), dst = smem_base + turn.s * stage_bytes;
                if (!wait_stage(empty(turn.s), turn.parity, abort_flag, p.err_word, kErrEmpty)) {
                    fine = false;
                    break;
                }
                mbar_arrive_expect_tx(bar, stage_bytes);
                if (wide) {
                    const int kq = k >= q.k_wrap ? k - q.k_wrap : k;
                    tma_load_2d_local(dst, &mw, (int)n0, kq, bar);
                    tma_load_2d_local(dst + 8192, &mw, (int)n0 + 64, kq, bar);
                } else {
                    tma_load_2d_local(dst, &mw, k, (int)n0, bar);
                }
                if (q.a_mn) {
                    tma_load_2d_local(dst + kOperandBytes, &mx, (int)m0, k, bar);
                    if (tokens > 64) tma_load_2d_local(dst + kOperandBytes + 8192, &mx, (int)m0 + 64, k, bar);
                } else {
                    tma_load_2d_local(dst + kOperandBytes, &mx, k, (int)m0, bar);
                }
            }
            if (!fine) {
                const long long t0 = clock64();
                while (clock64() - t0 < 2000000) {
                }
            }
        }
    } else if (warp == kSlimMma) {
        Turn turn{0, 0};
        const uint32_t idesc = instruction(128, tokens, q.b_mn, q.a_mn);
        const uint64_t w0 = operand(smem_base, q.b_mn), x0 = operand(smem_base + kOperandBytes, q.a_mn);
        const uint64_t w_next = q.b_mn ? kNextMn : kNextK, x_next = q.a_mn ? kNextMn : kNextK;
        uint32_t d = tmem_base, pass_n = 0;
        int begin = k_begin, end = SUMS == kFolded && k_end - k_begin > kFoldBlocks ? k_begin + kFoldBlocks : k_end;
        bool ready = false;
        for (int kb = k_begin; kb < k_end; ++kb) {
            if (SUMS == kFolded && kb == end) {   // the next accumulator, as in the kernel on pairs
                commit_elected_one(tmem_full(pass_n & 1));
                ++pass_n;
                const uint32_t acc = pass_n & 1, use = pass_n >> 1;
                if (use > 0 && !__all_sync(~0u, wait_stage(tmem_empty(acc), (use - 1) & 1, abort_flag, p.err_word, kErrTmemEmpty))) break;
                d = tmem_base + acc * each;
                begin = kb;
                end = k_end - kb > kFoldBlocks ? kb + kFoldBlocks : k_end;
            }
            if (!__all_sync(~0u, ready || wait_stage(full(turn.s), turn.parity, abort_flag, p.err_word, kErrFull))) break;
            tc_fence_after();
            const uint64_t at = (uint64_t)(turn.s * (stage_bytes >> 4));
            const uint32_t release = empty(turn.s);
            turn.next(stages);
            ready = kb + 1 < k_end && peek(full(turn.s), turn.parity);
#pragma unroll
            for (int k16 = 0; k16 < kBlockK / 16; ++k16)
                umma_elected_one(SUMS == kTwoSums ? d + ((kb - begin) & 1) * each : d, w0 + at + k16 * w_next, x0 + at + k16 * x_next, idesc,
                                 (kb > begin + (SUMS == kTwoSums) || k16 > 0) ? 1u : 0u);
            commit_elected_one(release);
        }
        commit_elected_one(tmem_full(pass_n & 1));
    }
    __syncwarp();
    // Epilogue warp w: lanes 32 (w mod 4) .., the first or the second half of the columns
    const int half = tokens < 32 ? 16 : tokens / 2, first = (warp >> 2) * half;
    const uint32_t taddr = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + first;
    float sum[SUMS == kFolded ? 4 : 1][16];
    if (warp < kSlimEpi) {
        mbar_wait_warp(tmem_full(0), 0, abort_flag, p.err_word, kErrTmemFull, lane);
        tc_fence_after();
        if constexpr (SUMS == kFolded) {   // the accumulators in turn
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int j = 0; j < 16; ++j) sum[c][j] = 0.f;
            uint32_t pass_n = 0;
            for (int left = k_end - k_begin;;) {
                const uint32_t acc = pass_n & 1;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (16 * c >= half || first >= tokens) break;   // the same for the whole warp
                    uint32_t w[16];
                    tmem_ld16(taddr + acc * each + 16 * c, w);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[c][j] += __uint_as_float(w[j]);
                }
                left -= kFoldBlocks;
                if (left <= 0) break;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(tmem_empty(acc));
                ++pass_n;
                if (!mbar_wait_warp(tmem_full(pass_n & 1), pass_n >> 1 & 1, abort_flag, p.err_word, kErrTmemFull, lane)) break;
                tc_fence_after();
            }
        }
    }
    // every CTA of the cluster has started: its shared memory may be written
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp < kSlimEpi) {
        const int end = (int)min((int64_t)min(tokens, first + half), q.rows - m0);   // columns behind the last token are not sent
        const int row = (warp & 3) * 32 + lane;
        const bool any = k_end > k_begin;
        const uint32_t part0 = smem_u32(part) + 4u * (rank * most * 128 + row);
        uint32_t owner = first % ranks, i = first / ranks;
        auto send = [&](int c0, const float (&v)[16]) {
            if (ranks == 1) {
#pragma unroll
                for (int j = 0; j < 16; ++j) part[(c0 + j) * 128 + row] = any ? v[j] : 0.f;
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (c0 + j < end) st_cluster(map_to_cta(part0 + 512u * i, owner), any ? v[j] : 0.f);
                    if (++owner == ranks) {
                        owner = 0;
                        ++i;
                    }
                }
            }
        };
        if constexpr (SUMS == kFolded) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (first + 16 * c < end) send(first + 16 * c, sum[c]);
        } else {
            for (int c0 = first; c0 < end; c0 += 16) {
                uint32_t w[16];
                tmem_ld16(taddr + c0 - first, w);
                tmem_ld_wait();
                float v[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(w[j]);
                if (SUMS == kTwoSums && k_end > k_begin + 1) {
                    tmem_ld16(taddr + each + c0 - first, w);
                    tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] += __uint_as_float(w[j]);
                }
                send(c0, v);
            }
        }
        tc_fence_before();
    }
    cluster_sync_all();
    if (warp < kSlimEpi) {
        switch (q.act) {
            case DASTAC_ACT_RELU: slim_finish<DASTAC_ACT_RELU>(q, part, tokens, ranks, rank, m0, n0, warp, lane); break;
            case DASTAC_ACT_SIGMOID: slim_finish<DASTAC_ACT_SIGMOID>(q, part, tokens, ranks, rank, m0, n0, warp, lane); break;
            case DASTAC_ACT_SILU: slim_finish<DASTAC_ACT_SILU>(q, part, tokens, ranks, rank, m0, n0, warp, lane); break;
            case DASTAC_ACT_GELU: slim_finish<DASTAC_ACT_GELU>(q, part, tokens, ranks, rank, m0, n0, warp, lane); break;
            default: slim_finish<DASTAC_ACT_NONE>(q, part, tokens, ranks, rank, m0, n0, warp, lane); break;
        }
    } else if (warp == kSlimMma) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc_one(tmem_base, tmem_cols);
    }
}

// ---- preparing operands ------------------------------------------------------------------------------------
// A copy with a pitch that a tensor map can describe; eight elements a thread, the pad zero.
__global__ void linear_repitch_kernel(const uint16_t* __restrict__ src, int64_t lds, uint16_t* __restrict__ dst, int64_t ldd,
                                      int64_t rows, int64_t cols) {
    const int64_t per_row = ldd / 8;
    for (int64_t t = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; t < rows * per_row; t += (int64_t)gridDim.x * blockDim.x) {
        const int64_t r = t / per_row, c = (t - r * per_row) * 8;
        union {
            uint16_t h[8];
            uint4 q;
        } v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v.h[j] = c + j < cols ? src[r * lds + c + j] : (uint16_t)0;
        *(uint4*)(dst + r * ldd + c) = v.q;
    }
}

// dZ = dY f'(Z), rounded to bf16 for the products, where asked for also what that rounding leaves, rounded likewise, and
// the column sums of the unrounded values over 64 rows; VEC = 8: rows of whole aligned 16-byte words.  Bound by memory: a warp has four rows in flight.  The sums of the row
// blocks are added by a second kernel in a fixed order.
constexpr int kSumRows = 64;
struct SlopeParams {
    const __nv_bfloat16* dy;
    int64_t lddy;
    const __nv_bfloat16* z;
    int64_t ldz;
    __nv_bfloat16* dz;   // NULL: sums only
    __nv_bfloat16* rest; // dZ - dz, where REST: rows in whole blocks of kSumRows, behind those of dz, what lies beyond M zero
    int64_t lddz;        // of both
    float* sums;         // [row blocks][N], NULL: none
    int64_t M, N;
};

template <int ACT, int VEC, bool REST>
__global__ void __launch_bounds__(256) linear_slope_kernel(const SlopeParams p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c = (int64_t)blockIdx.x * 32 * VEC + lane * VEC;
    const int64_t r0 = (int64_t)blockIdx.y * kSumRows;
    float sum[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
    union Word {
        uint4 q;
        __nv_bfloat16 h[8];
    };
    if (c < p.N) {
        constexpr int kAtOnce = 4;   // rows whose loads are in flight together
#pragma unroll 1
        for (int i = warp; i < kSumRows; i += 8 * kAtOnce) {
            Word dy[kAtOnce], z[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int64_t r = r0 + i + 8 * k;
                dy[k].q = z[k].q = make_uint4(0, 0, 0, 0);
                if (r < p.M) {
                    if (VEC == 8) {
                        dy[k].q = *(const uint4*)(p.dy + r * p.lddy + c);
                        if (ACT != DASTAC_ACT_NONE) z[k].q = *(const uint4*)(p.z + r * p.ldz + c);
                    } else {
                        dy[k].h[0] = p.dy[r * p.lddy + c];
                        if (ACT != DASTAC_ACT_NONE) z[k].h[0] = p.z[r * p.ldz + c];
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int64_t r = r0 + i + 8 * k;
                Word o, rest;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    float v = __bfloat162float(dy[k].h[j]);
                    if (ACT != DASTAC_ACT_NONE) v *= slope_of<ACT>(__bfloat162float(z[k].h[j]));
                    if (r < p.M) sum[j] += v;
                    o.h[j] = __float2bfloat16_rn(v);
                    // an infinity leaves nothing (and not NaN)
                    if (REST) rest.h[j] = __float2bfloat16_rn((__bfloat16_as_ushort(o.h[j]) & 0x7f80) == 0x7f80 ? 0.f : v - __bfloat162float(o.h[j]));
                }
                if (p.dz && (REST || r < p.M)) {
                    if (VEC == 8) *(uint4*)(p.dz + r * p.lddz + c) = o.q;
                    else p.dz[r * p.lddz + c] = o.h[0];
                }
                if (REST) {
                    if (VEC == 8) *(uint4*)(p.rest + r * p.lddz + c) = rest.q;
                    else p.rest[r * p.lddz + c] = rest.h[0];
                }
            }
        }
    }
    if (!p.sums) return;
    __shared__ float part[8][32 * VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) part[warp][lane * VEC + j] = sum[j];
    __syncthreads();
    for (int t = threadIdx.x; t < 32 * VEC; t += 256) {
        const int64_t n = (int64_t)blockIdx.x * 32 * VEC + t;
        if (n < p.N) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) v += part[w][t];
            p.sums[blockIdx.y * p.N + n] = v;
        }
    }
}

__global__ void linear_column_sum_kernel(const float* __restrict__ sums, int64_t blocks, int64_t N, float* db, int accumulate) {
    // a block of 32 columns, eight partial sums a column, joined in a fixed order
    __shared__ float part[8][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t n = (int64_t)blockIdx.x * 32 + lane;
    float v = 0.f;
    if (n < N)
        for (int64_t b = warp; b < blocks; b += 8) v += sums[b * N + n];
    part[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && n < N) {
        v = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) v += part[w][lane];
        db[n] = accumulate ? db[n] + v : v;
    }
}

// ---- host --------------------------------------------------------------------------------------------------
constexpr int64_t kMaxExtent = (int64_t)1 << 30;

bool map_ok(const void* p, int64_t ld) { return aligned16(p) && ld % 8 == 0; }

// A tensor map of a rows x cols bf16 matrix with boxes of `box_rows` x 64 elements.
bool encode(CUtensorMap* m, const void* p, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? ld : round_up(cols, 8)) * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Operand {
    const void* p;
    int64_t rows, cols, ld;
    bool staged;  // copied into the workspace first
    size_t at;    // where
};
Operand operand_of(const void* p, int64_t rows, int64_t cols, int64_t ld, size_t& bytes) {
    Operand o{p, rows, cols, ld, rows > 0 && cols > 0 && !(aligned16(p) && (rows <= 1 || ld % 8 == 0)), bytes};
    if (o.staged) bytes += (size_t)round_up(rows * round_up(cols, 8) * 2, 256);
    return o;
}
dastac_status stage(Operand& o, void* workspace, cudaStream_t st) {
    if (!o.staged) return DASTAC_OK;
    const int64_t ldd = round_up(o.cols, 8);
    uint16_t* dst = (uint16_t*)((char*)workspace + o.at);
    const int64_t blocks = (o.rows * (ldd / 8) + 255) / 256, most = (int64_t)sm_count() * 16;
    linear_repitch_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, st>>>((const uint16_t*)o.p, o.ld, dst, ldd, o.rows, o.cols);
    o.p = dst;
    o.ld = ldd;
    return launch_status();
}

dastac_status check_common(const dastac_linear_args* a) {
    if (!a || a->M < 0 || a->N < 0 || a->K < 0) return DASTAC_ERR_INVALID_ARG;
    if (a->M > kMaxExtent || a->N > kMaxExtent || a->K > kMaxExtent) return DASTAC_ERR_OVERFLOW;
    if (a->act < DASTAC_ACT_NONE || a->act > DASTAC_ACT_GELU) return DASTAC_ERR_INVALID_ARG;
    return DASTAC_OK;
}
// A row-major matrix argument: present, whole elements, rows that do not overlap.
dastac_status check_matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, int elt) {
    if (rows == 0 || cols == 0) return DASTAC_OK;
    if (!p) return DASTAC_ERR_INVALID_ARG;
    if (rows > 1 && ld < cols) return DASTAC_ERR_SHAPE;
    if ((uintptr_t)p % elt) return DASTAC_ERR_ALIGNMENT;
    return DASTAC_OK;
}
dastac_status check_forward(const dastac_linear_args* a) {
    dastac_status st = check_common(a);
    if (st != DASTAC_OK) return st;
    if (a->y_dtype != DASTAC_F32 && a->y_dtype != DASTAC_BF16) return DASTAC_ERR_UNSUPPORTED_EXPR;
    const int e = elt_size(a->y_dtype);
    if (a->M == 0 || a->N == 0) return DASTAC_OK;
    if ((st = check_matrix(a->x, a->M, a->K, a->ldx, 2)) != DASTAC_OK || (st = check_matrix(a->w, a->N, a->K, a->ldw, 2)) != DASTAC_OK ||
        (st = check_matrix(a->y, a->M, a->N, a->ldy, e)) != DASTAC_OK)
        return st;
    if (a->residual && (st = check_matrix(a->residual, a->M, a->N, a->ldr, e)) != DASTAC_OK) return st;
    if (a->z && (st = check_matrix(a->z, a->M, a->N, a->ldz, 2)) != DASTAC_OK) return st;
    if ((uintptr_t)a->bias & 3) return DASTAC_ERR_ALIGNMENT;
    return DASTAC_OK;
}
dastac_status check_backward(const dastac_linear_args* a) {
    dastac_status st = check_common(a);
    if (st != DASTAC_OK) return st;
    if (a->dw && a->dw_dtype != DASTAC_F32 && a->dw_dtype != DASTAC_BF16) return DASTAC_ERR_UNSUPPORTED_EXPR;
    if (a->dw && a->accumulate && a->dw_dtype != DASTAC_F32) return DASTAC_ERR_UNSUPPORTED_EXPR;
    if ((st = check_matrix(a->dy, a->M, a->N, a->lddy, 2)) != DASTAC_OK) return st;
    if (a->act != DASTAC_ACT_NONE && (st = check_matrix(a->z, a->M, a->N, a->ldz, 2)) != DASTAC_OK) return st;
    if (a->dx && ((st = check_matrix(a->w, a->N, a->K, a->ldw, 2)) != DASTAC_OK || (st = check_matrix(a->dx, a->M, a->K, a->lddx, 2)) != DASTAC_OK))
        return st;
    if (a->dw && ((st = check_matrix(a->x, a->M, a->K, a->ldx, 2)) != DASTAC_OK ||
                  (st = check_matrix(a->dw, a->N, a->K, a->lddw, elt_size(a->dw_dtype))) != DASTAC_OK))
        return st;
    if ((uintptr_t)a->db & 3) return DASTAC_ERR_ALIGNMENT;
    return DASTAC_OK;
}

// Whether `bytes` bytes at the beginning of every row are aligned to as many.
bool row_aligned(const void* p, int64_t ld, int elt, int bytes) { return !p || ((uintptr_t)p % bytes == 0 && ld * elt % bytes == 0); }
void set_alignment(Problem& q) {
    const int e = elt_size(q.out_dtype);
    auto all = [&](int out, int z) {
        return row_aligned(q.out, q.ld, e, out) && row_aligned(q.residual, q.ldr, e, out) && row_aligned(q.z, q.ldz, 2, z);
    };
    q.even = all(2 * e, 4);
    q.quad = all(4 * e, 8);
    q.whole = all(16, 16);
    q.wide = all(32, 32);
}

Problem problem_of(int a_mn, int b_mn, int64_t rows, int64_t cols, int64_t k, void* out, int64_t ld, int out_dtype) {
    Problem q{};
    q.a_mn = a_mn;
    q.b_mn = b_mn;
    q.rows = rows;
    q.cols = cols;
    q.k_blocks = (int32_t)((k + kBlockK - 1) / kBlockK);
    q.k_wrap = INT32_MAX;
    q.row_blocks = (int32_t)((rows + 255) / 256);
    q.col_blocks = (int32_t)((cols + 255) / 256);
    q.act = DASTAC_ACT_NONE;
    q.out = out;
    q.ld = ld;
    q.out_dtype = out_dtype;
    return q;
}

int64_t tiles_of(const Problem& q) { return (int64_t)q.row_blocks * q.col_blocks; }

struct Maps {
    CUtensorMap a, b;
};
bool encode_problem(const Problem& q, const Operand& P, const Operand& Q, Maps& m) {
    if (q.k_blocks == 0) return true;
    return encode(&m.a, P.p, P.rows, P.cols, P.ld, q.a_mn ? 64 : 128) && encode(&m.b, Q.p, Q.rows, Q.cols, Q.ld, q.b_mn ? 64 : 128);
}

bool set_smem_once(const void* kernel, size_t bytes, bool* done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if (!done[dev]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return false;
        done[dev] = true;
    }
    return true;
}

template <bool DIRECT, bool FOLD>
dastac_status launch_pair_as(const PairParams& p, const Maps& m0, const Maps& m1, cudaStream_t st) {
    static bool attr[64];
    if (!set_smem_once((const void*)linear_pair_kernel<DIRECT, FOLD>, kPairSmem<DIRECT>, attr)) return DASTAC_ERR_CUDA;
    const int64_t most = sm_count() / 2;
    const int clusters = (int)(p.tiles < most ? p.tiles : most);
    linear_pair_kernel<DIRECT, FOLD><<<2 * clusters, kPairThreads, kPairSmem<DIRECT>, st>>>(m0.a, m0.b, m1.a, m1.b, p);
    return launch_status();
}
dastac_status launch_pair(const Problem* q, const Maps* m, int n, int32_t* err_word, cudaStream_t st) {
    PairParams p{};
    p.q[0] = q[0];
    p.q[1] = q[n - 1];
    p.tiles0 = tiles_of(q[0]);
    p.tiles = p.tiles0 + (n > 1 ? tiles_of(q[1]) : 0);
    p.err_word = err_word;
    for (Problem& one : p.q) one.fold = one.out_dtype == DASTAC_F32 && one.k_blocks > kFoldBlocks;
    const bool direct = q[0].whole && q[n - 1].whole;
    if (p.q[0].fold || p.q[1].fold)
        return direct ? launch_pair_as<true, true>(p, m[0], m[n - 1], st) : launch_pair_as<false, true>(p, m[0], m[n - 1], st);
    return direct ? launch_pair_as<true, false>(p, m[0], m[n - 1], st) : launch_pair_as<false, false>(p, m[0], m[n - 1], st);
}

// CTAs of the slim kernel that the device holds at once in clusters of `ranks`, `per_sm` on a multiprocessor: clusters have
// to fit into its groups of multiprocessors (of eight, one to an SM: 120 CTAs, not 148).
int64_t slim_slots(int dev, int sms, int ranks, int per_sm) {
    static int cached[64][9][8];
    const int64_t guess = (int64_t)sms * per_sm;
    if (per_sm > 7) return guess;
    int& n = cached[dev][ranks][per_sm];
    if (n == 0) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(64 * ranks), 1, 1);
        cfg.blockDim = dim3(kSlimThreads, 1, 1);
        cfg.dynamicSmemBytes = (233472 / per_sm - 1024) / 1024 * 1024;
        if (cfg.dynamicSmemBytes > kSlimMax + 2048) cfg.dynamicSmemBytes = kSlimMax + 2048;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = (unsigned)ranks;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, linear_slim_kernel<kOneSum>, &cfg) != cudaSuccess || clusters <= 0) {
            cudaGetLastError();
            return guess;
        }
        n = clusters * ranks;
    }
    return n;
}

// Which kernel, and how the slim one is laid out: by the time, in us, that each is expected to take.  The constants
// are fitted to 72 shapes (1 .. 800 rows, 384 .. 8192 columns, 320 .. 8192 inner), each with every layout: the layout
// picked is within 0.4 % of the fastest in the mean, 5 % at the worst.  With 4096 x 4096 weights slim takes 11 us (24
// rows), 13.8 (100) and 17.5 (200) against 25.6 to 26.7 for the pairs; at 512 rows, 26.1 and 27.5, the two meet.
struct SlimPlan {
    int tokens, ranks, stages;
    size_t smem;
    double us;
};
SlimPlan lay_out_slim(const Problem& q, int dev, int sms, int tokens, int ranks) {
    SlimPlan l{tokens, ranks, 0, 0, 0.0};
    const size_t stage_bytes = kOperandBytes + (size_t)tokens * kBlockK * 2;
    const size_t part = (size_t)ranks * ((tokens + ranks - 1) / ranks) * 128 * 4;
    const int64_t longest = (q.k_blocks + ranks - 1) / ranks, fit = (int64_t)((kSlimMax - part) / stage_bytes);
    l.stages = (int)(fit < longest ? fit : longest < 1 ? 1 : longest);
    l.smem = 1024 + l.stages * stage_bytes + part + 16 * (size_t)l.stages + 64;
    // Never on one SM with a CTA of the kernels on pairs, which hold all of the tensor memory: two kernels
    // whose clusters wait for their own CTAs must not also wait for each other's tensor memory.  CTAs of this
    // kernel that fit on an SM together never ask for more than there is: 256 columns come with at least 98 KB of
    // shared memory, 128 with 58, 64 with 41, and no such sum within 228 KB passes 512 columns.
    if (l.smem < kSlimLeast) l.smem = kSlimLeast;
    const int64_t ctas = (q.cols + 127) / 128 * ((q.rows + tokens - 1) / tokens) * ranks;
    const int64_t slots = slim_slots(dev, sms, ranks, (int)(233472 / (l.smem + 1024)));
    const double waves = (double)((ctas + slots - 1) / slots), busy = (double)(ctas < slots ? ctas : slots);
    // MB a us that so many CTAs draw from memory; a stage every 0.27 us, less often where CTAs share an SM
    const double drawn = 0.084 * (busy < sms ? busy : sms), rate = drawn < 7.7 ? drawn : 7.7;
    const double load = 128e-6 * q.k_blocks * ((double)q.cols + q.rows) / waves / rate, multiply = (busy > sms ? 0.85 : 0.272) * longest;
    l.us = 1.1 + waves * (2.84 + (load > multiply ? load : multiply) + tokens * (0.0166 + 0.02 / ranks) + (ranks > 1 ? 0.39 : 0.0));
    return l;
}
SlimPlan plan_slim(const Problem& q) {
    SlimPlan best{0, 1, 1, 0, 1e30};
    static bool attr[3][64];
    int dev = 0;
    if (!set_smem_once((const void*)linear_slim_kernel<kOneSum>, kSlimMax + 2048, attr[kOneSum]) ||
        !set_smem_once((const void*)linear_slim_kernel<kTwoSums>, kSlimMax + 2048, attr[kTwoSums]) ||
        !set_smem_once((const void*)linear_slim_kernel<kFolded>, kSlimMax + 2048, attr[kFolded]) || cudaGetDevice(&dev) != cudaSuccess) return best;
    const int sms = sm_count();
    const int least = q.a_mn ? 64 : 16;
    for (int t = least; t <= 128; t *= 2) {
        if (t > least && q.rows <= t / 2) break;            // half of the columns would be empty
        if (t < 64 && q.rows > t) continue;                 // narrow tiles only where one holds all tokens
        for (int r = 1; r <= 8; ++r) {
            if (r > 1 && 2 * r > q.k_blocks) break;
            const SlimPlan l = lay_out_slim(q, dev, sms, t, r);
            if (l.us < best.us) best = l;
        }
    }
    return best;
}
// The kernel on pairs, for n products in one launch: whole rounds of tiles for one product; two fill each other's gaps.
double pair_us(const Problem* q, int n) {
    const double clusters = sm_count() / 2;
    double work = 0.0, longest = 0.0;
    bool whole = true, wide = true;
    for (int i = 0; i < n; ++i) {
        const double tile = q[i].k_blocks * 0.278 + 1.0;
        work += (double)tiles_of(q[i]) * tile;
        if (tile > longest) longest = tile;
        whole = whole && q[i].whole;
        wide = wide && q[i].wide;
    }
    double busy = work / clusters + 0.4 * longest;
    if (n == 1) busy = (double)((tiles_of(q[0]) + (int64_t)clusters - 1) / (int64_t)clusters) * longest;
    if (busy < longest) busy = longest;
    return 7.3 + busy + (!whole ? 5.0 : !wide ? 2.5 : 0.0);
}

dastac_status launch_slim(const SlimPlan& plan, const Problem& q, const Operand& W, const Operand& X, int32_t* err_word, cudaStream_t st) {
    const int ranks = plan.ranks;
    SlimParams p{};
    p.q = q;
    p.tokens = plan.tokens;
    p.stages = plan.stages;
    p.err_word = err_word;
    const int64_t n_tiles = (q.cols + 127) / 128, m_tiles = (q.rows + p.tokens - 1) / p.tokens;
    if (m_tiles > 65535) return DASTAC_ERR_OVERFLOW;
    CUtensorMap mw{}, mx{};
    if (q.k_blocks && (!encode(&mw, W.p, W.rows, W.cols, W.ld, q.b_mn ? 64 : 128) || !encode(&mx, X.p, X.rows, X.cols, X.ld, q.a_mn ? 64 : p.tokens)))
        return DASTAC_ERR_CUDA;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(n_tiles * ranks), (unsigned)m_tiles, 1);
    cfg.blockDim = dim3(kSlimThreads, 1, 1);
    cfg.dynamicSmemBytes = plan.smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)ranks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const bool few = q.out_dtype != DASTAC_F32 || q.k_blocks <= 1, folded = q.k_blocks > 2 * kFoldBlocks * ranks;   // some CTA has more blocks than two accumulators take
    auto kernel = few ? linear_slim_kernel<kOneSum> : folded ? linear_slim_kernel<kFolded> : linear_slim_kernel<kTwoSums>;
    if (cudaLaunchKernelEx(&cfg, kernel, mw, mx, p) != cudaSuccess) {
        cudaGetLastError();
        return DASTAC_ERR_CUDA;
    }
    return launch_status();
}

bool on_pairs(const Problem& q, const SlimPlan& slim) { return slim.us >= pair_us(&q, 1); }
dastac_status multiply(const Problem& q, const Operand& P, const Operand& Q, int32_t* err_word, cudaStream_t st) {
    const SlimPlan plan = plan_slim(q);
    if (!on_pairs(q, plan)) return launch_slim(plan, q, Q, P, err_word, st);
    Maps m{};
    if (!encode_problem(q, P, Q, m)) return DASTAC_ERR_CUDA;
    return launch_pair(&q, &m, 1, err_word, st);
}

template <int VEC, bool REST>
void launch_slope_as(const SlopeParams& p, int act, cudaStream_t st) {
    const dim3 grid((unsigned)((p.N + 32 * VEC - 1) / (32 * VEC)), (unsigned)((p.M + kSumRows - 1) / kSumRows));
    switch (act) {
        case DASTAC_ACT_SIGMOID: linear_slope_kernel<DASTAC_ACT_SIGMOID, VEC, REST><<<grid, 256, 0, st>>>(p); break;
        case DASTAC_ACT_SILU: linear_slope_kernel<DASTAC_ACT_SILU, VEC, REST><<<grid, 256, 0, st>>>(p); break;
        case DASTAC_ACT_GELU: linear_slope_kernel<DASTAC_ACT_GELU, VEC, REST><<<grid, 256, 0, st>>>(p); break;
        // no rest where dZ is dY or 0
        case DASTAC_ACT_RELU: linear_slope_kernel<DASTAC_ACT_RELU, VEC, false><<<grid, 256, 0, st>>>(p); break;
        default: linear_slope_kernel<DASTAC_ACT_NONE, VEC, false><<<grid, 256, 0, st>>>(p); break;
    }
}
template <int VEC>
void launch_slope(const SlopeParams& p, int act, cudaStream_t st) {
    if (p.rest) launch_slope_as<VEC, true>(p, act, st);
    else launch_slope_as<VEC, false>(p, act, st);
}

// Where the backward pass keeps things: dZ (with an activation, or when dY is no operand as it lies) and what rounding it
// leaves, the partial column sums, copies of X and W.
//
// With an activation dZ has more bits than an operand of the products holds.  dX and a bf16 dW are rounded as coarsely
// themselves and take it rounded.  An fp32 dW would have that rounding's error (1.7e-3 of the result, 2048 rows), so its sum
// goes on over what the rounding leaves, a second part of dZ behind the first, with the same rows of X, unless the caller
// does without: 2.6e-6 (4096 rows, 4096 by 8192, SiLU, dX and dW: 650 us, 458 without; as a product of its own that is
// added to dW: 734).  relu's dZ is dY or 0 and needs none.
struct BackwardPlan {
    Operand x, w, dz;
    bool make_dz, make_rest;
    size_t dz_at, sums_at, bytes;
    int64_t row_blocks;
};
BackwardPlan plan_backward(const dastac_linear_args* a) {
    BackwardPlan b{};
    const bool products = (a->dx || a->dw) && a->K > 0;
    b.make_dz = products && (a->act != DASTAC_ACT_NONE || !(aligned16(a->dy) && (a->M <= 1 || a->lddy % 8 == 0)));
    b.make_rest = a->dw && a->K > 0 && a->act != DASTAC_ACT_NONE && a->act != DASTAC_ACT_RELU && a->dw_dtype == DASTAC_F32 && !a->round_dz;
    b.row_blocks = (a->M + kSumRows - 1) / kSumRows;
    b.dz = Operand{a->dy, a->M, a->N, a->lddy, false, 0};
    if (b.make_dz) {
        b.dz.ld = round_up(a->N, 8);
        b.dz_at = b.bytes;
        b.bytes += (size_t)round_up((b.make_rest ? 2 * b.row_blocks * kSumRows : a->M) * b.dz.ld * 2, 256);
    }
    b.sums_at = b.bytes;
    if (a->db) b.bytes += (size_t)round_up(b.row_blocks * a->N * 4, 256);
    b.w = operand_of(a->w, a->dx ? a->N : 0, a->K, a->ldw, b.bytes);
    b.x = operand_of(a->x, a->dw ? a->M : 0, a->K, a->ldx, b.bytes);
    return b;
}

Problem forward_problem(const dastac_linear_args* a) {
    Problem q = problem_of(0, 0, a->M, a->N, a->K, a->y, a->ldy, a->y_dtype);
    q.act = a->act;
    q.bias = a->bias;
    q.residual = a->residual;
    q.ldr = a->ldr;
    q.z = (__nv_bfloat16*)a->z;
    q.ldz = a->ldz;
    set_alignment(q);
    return q;
}

bool workspace_ok(size_t need, const void* w, size_t have) { return need == 0 || (w && have >= need && ((uintptr_t)w & 255) == 0); }

}  // namespace
}  // namespace dastac

using namespace dastac;

extern "C" dastac_status dastac_linear_forward_workspace(const dastac_linear_args* a, size_t* bytes) {
    const dastac_status st = check_forward(a);
    if (st != DASTAC_OK) return st;
    if (!bytes) return DASTAC_ERR_INVALID_ARG;
    *bytes = 0;
    if (a->M == 0 || a->N == 0) return DASTAC_OK;
    operand_of(a->x, a->M, a->K, a->ldx, *bytes);
    operand_of(a->w, a->N, a->K, a->ldw, *bytes);
    return DASTAC_OK;
}

extern "C" dastac_status dastac_linear_forward(const dastac_linear_args* a, void* workspace, size_t workspace_bytes,
                                               int32_t* err_word, void* stream) {
    dastac_status st = check_forward(a);
    if (st != DASTAC_OK) return st;
    if (a->M == 0 || a->N == 0) return DASTAC_OK;
    size_t need = 0;
    Operand x = operand_of(a->x, a->M, a->K, a->ldx, need), w = operand_of(a->w, a->N, a->K, a->ldw, need);
    if (!workspace_ok(need, workspace, workspace_bytes)) return DASTAC_ERR_WORKSPACE;
    cudaStream_t cs = (cudaStream_t)stream;
    if ((st = stage(x, workspace, cs)) != DASTAC_OK || (st = stage(w, workspace, cs)) != DASTAC_OK) return st;
    return multiply(forward_problem(a), x, w, err_word ? err_word : device_error_word(), cs);
}

extern "C" dastac_status dastac_linear_forward_kernel(const dastac_linear_args* a, int32_t* kernel) {
    const dastac_status st = check_forward(a);
    if (st != DASTAC_OK) return st;
    if (!kernel) return DASTAC_ERR_INVALID_ARG;
    *kernel = 0;
    if (a->M == 0 || a->N == 0) return DASTAC_OK;
    const Problem q = forward_problem(a);
    *kernel = on_pairs(q, plan_slim(q)) ? 2 : 1;
    return DASTAC_OK;
}

extern "C" dastac_status dastac_linear_backward_workspace(const dastac_linear_args* a, size_t* bytes) {
    const dastac_status st = check_backward(a);
    if (st != DASTAC_OK) return st;
    if (!bytes) return DASTAC_ERR_INVALID_ARG;
    *bytes = a->M == 0 || a->N == 0 ? 0 : plan_backward(a).bytes;
    return DASTAC_OK;
}

extern "C" dastac_status dastac_linear_backward(const dastac_linear_args* a, void* workspace, size_t workspace_bytes,
                                                int32_t* err_word, void* stream) {
    dastac_status st = check_backward(a);
    if (st != DASTAC_OK) return st;
    cudaStream_t cs = (cudaStream_t)stream;
    if (a->M == 0 || a->N == 0) {   // empty sums
        if (a->dx && a->M > 0 && a->K > 0 && cudaMemset2DAsync(a->dx, (size_t)a->lddx * 2, 0, (size_t)a->K * 2, (size_t)a->M, cs) != cudaSuccess)
            return DASTAC_ERR_CUDA;
        if (a->accumulate || a->N == 0) return DASTAC_OK;
        const int e = elt_size(a->dw_dtype);
        if (a->dw && a->K > 0 && cudaMemset2DAsync(a->dw, (size_t)a->lddw * e, 0, (size_t)a->K * e, (size_t)a->N, cs) != cudaSuccess)
            return DASTAC_ERR_CUDA;
        if (a->db && cudaMemsetAsync(a->db, 0, (size_t)a->N * 4, cs) != cudaSuccess) return DASTAC_ERR_CUDA;
        return DASTAC_OK;
    }
    BackwardPlan b = plan_backward(a);
    if (!workspace_ok(b.bytes, workspace, workspace_bytes)) return DASTAC_ERR_WORKSPACE;
    if (b.row_blocks > 65535) return DASTAC_ERR_OVERFLOW;   // gridDim.y of the slope kernel
    if (b.make_dz || a->db) {
        SlopeParams s{};
        s.dy = (const __nv_bfloat16*)a->dy;
        s.lddy = a->lddy;
        s.z = (const __nv_bfloat16*)a->z;
        s.ldz = a->ldz;
        s.dz = b.make_dz ? (__nv_bfloat16*)((char*)workspace + b.dz_at) : nullptr;
        s.rest = b.make_rest ? s.dz + b.row_blocks * kSumRows * b.dz.ld : nullptr;
        s.lddz = b.dz.ld;
        s.sums = a->db ? (float*)((char*)workspace + b.sums_at) : nullptr;
        s.M = a->M;
        s.N = a->N;
        const bool wide = a->N % 8 == 0 && map_ok(a->dy, a->lddy) && (a->act == DASTAC_ACT_NONE || map_ok(a->z, a->ldz));
        if (wide) launch_slope<8>(s, a->act, cs);
        else launch_slope<1>(s, a->act, cs);
        if ((st = launch_status()) != DASTAC_OK) return st;
        if (b.make_dz) b.dz.p = s.dz;
        if (a->db) {
            linear_column_sum_kernel<<<(unsigned)((a->N + 31) / 32), 256, 0, cs>>>(s.sums, b.row_blocks, a->N, a->db, a->accumulate);
            if ((st = launch_status()) != DASTAC_OK) return st;
        }
    }
    if (a->K == 0 || (!a->dx && !a->dw)) return DASTAC_OK;
    if ((st = stage(b.w, workspace, cs)) != DASTAC_OK || (st = stage(b.x, workspace, cs)) != DASTAC_OK) return st;
    if (!err_word) err_word = device_error_word();
    Problem q[2];
    Operand P[2], Q[2];
    int n = 0;
    if (a->dx) {
        q[n] = problem_of(0, 1, a->M, a->K, a->N, a->dx, a->lddx, DASTAC_BF16);
        P[n] = b.dz;
        Q[n++] = b.w;
    }
    if (a->dw) {
        static_assert(kSumRows % kBlockK == 0, "the second part begins with a block of k");
        const int64_t part = b.row_blocks * kSumRows;
        q[n] = problem_of(1, 1, a->N, a->K, b.make_rest ? 2 * part : a->M, a->dw, a->lddw, a->dw_dtype);
        q[n].accumulate = a->accumulate;
        P[n] = b.dz;
        if (b.make_rest) {
            P[n].rows = 2 * part;
            q[n].k_wrap = (int32_t)part;
        }
        Q[n++] = b.x;
    }
    // each by itself, whichever kernel suits it, or both in one launch on the pairs (2001 rows, 520 by 1363: on the GPU
    // all of it takes 36 us with one launch of products, 41.5 with two; 4096 rows, 4096 by 8192: 412 and 424)
    double apart = 0.0;
    for (int i = 0; i < n; ++i) {
        set_alignment(q[i]);
        const double slim = plan_slim(q[i]).us, pair = pair_us(&q[i], 1);
        apart += slim < pair ? slim : pair;
    }
    if (n < 2 || apart < pair_us(q, n)) {
        for (int i = 0; i < n; ++i)
            if ((st = multiply(q[i], P[i], Q[i], err_word, cs)) != DASTAC_OK) return st;
        return DASTAC_OK;
    }
    Maps m[2]{};
    for (int i = 0; i < 2; ++i)
        if (!encode_problem(q[i], P[i], Q[i], m[i])) return DASTAC_ERR_CUDA;
    if (q[1].k_blocks > q[0].k_blocks) {   // the longer contraction first
        const Problem tq = q[0];
        const Maps tm = m[0];
        q[0] = q[1];
        m[0] = m[1];
        q[1] = tq;
        m[1] = tm;
    }
    return launch_pair(q, m, 2, err_word, cs);
}
