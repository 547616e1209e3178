// es_q8_grad.h -- dW = X^T G with X held as 8-bit rows: the weight gradient of a dense layer from its input's checkpoint.
//
//   dW[i, j] = sum over r of code[r, i] * (scale[r] * G[r, j])
//
// On the matrix cores in bf16, exactly: a code has 8 significant bits and is a bf16 number; g = scale * G, rounded once to
// fp32, is the sum of three bf16 numbers, its leading, middle and last 8 bits (exactly from |g| of 2^-110 on; bf16 ends at
// 2^-133, and bits of g below that are lost); every product of the two is exact in fp32.  What is rounded is g and the sums, in fp32.
//
// A matrix instruction wants 8 rows r of one column i (or j) in a lane's registers, and in memory a row's columns lie
// side by side.  No data has to be turned for that: a lane loads the same 4 columns of codes (2 of G) of 8 rows, and
// registers number c of those loads are what the lane owes the c-th of 4 (2) tiles; which 32 columns
// a tile then has, every fourth (second), is of no consequence until the result is stored.  A narrow dW takes fewer tiles.
//
// 233 k rows, 602 x 256: 250 us and 9 us of join, 0.86 PFLOP/s of the three products.  Of its 548 k clocks (2.14 GHz) the matrix cores
// are busy for 40 %, and the vector ALUs, which convert and split the operands, for about as many; 10 % of the waves' time is waiting for
// memory.  That is most of the time if the two waves of a SIMD overlap the one with the other as little as it looks; the matrix cores' rate
// alone does not bound it (a library's bf16 product of 8192^3: 69 % at 1.69 GHz).  2.45 M rows, 128 x 128: 280 us and 4 us, bound by HBM (5.2
// TB/s).
#ifndef ES_SPMM_Q8_GRAD_H
#define ES_SPMM_Q8_GRAD_H

#include "es_common.h"

namespace {

struct Q8Grad {
    const int8_t* codes;
    const float* scale;
    const float* G;
    float* dW;                 // the result, or the parts' sums
    int64_t N;
    int32_t F, H, ldq, ldg, ldw;
    int32_t tiles_m, tiles;    // tiles of dW: along F, and in all
    int64_t part_rows;         // rows of X that one part sums
    int32_t parts;
};

constexpr int kGradTile = 32;                                  // rows and columns of dW of an instruction
constexpr int kGradStep = 16;                                  // rows of X that an instruction sums
constexpr int kGradRows = kGradStep * kWavesPerBlock;          // ... and a workgroup's four waves together

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float float4_u4 __attribute__((ext_vector_type(4), aligned(4)));

// One load of MT codes or of NT numbers of G, at any alignment.
template <int MT> struct GradCodes;
template <> struct GradCodes<1> { typedef uint8_t type; };
template <> struct GradCodes<2> { typedef uint16_t type; };
template <> struct GradCodes<4> { typedef uint32_t type; };
template <int NT> struct GradPair { typedef float type __attribute__((ext_vector_type(NT), aligned(4))); };

// What a lane loads of 8 rows.
template <int NT>
struct GradRows {
    uint32_t code[8];
    float g[8][NT];
    float4_u4 scale[2];
};

// the upper halves of two words: numbers cut to bf16
__device__ __forceinline__ uint32_t upper_halves(float low, float high)
{
    return __builtin_amdgcn_perm(__float_as_uint(high), __float_as_uint(low), 0x07060302u);
}
union GradFrag { uint32_t w[4]; bf16x8 v; };

// The four waves of a workgroup take the part's steps in turn and add up their tiles in LDS, in their order.
// A wave's tile of dW is MT x NT tiles of the instruction.
template <int MT, int NT>
__global__ void __launch_bounds__(kBlockThreads, 2) es_q8_grad_kernel(const Q8Grad a)
{
    constexpr int M = MT * kGradTile, N = NT * kGradTile;
    __shared__ float sums[2][M * N];
    const int lane = threadIdx.x & (kWaveSize - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, half = lane >> 5;
    // the tiles of a part run on one XCD: they read the same rows
    const uint32_t groups = a.parts < kNumXcd ? 1 : kNumXcd;
    const uint32_t i = blockIdx.x / groups;
    const int32_t part = (int32_t)(i / a.tiles * groups + blockIdx.x % groups), tile = (int32_t)(i % a.tiles);
    if (part >= a.parts) return;
    const int32_t m0 = tile % a.tiles_m * M, n0 = tile / a.tiles_m * N;
    const int64_t lo = part * a.part_rows, hi = min(a.N, lo + a.part_rows);
    const int32_t cm = m0 + MT * n, cn = n0 + NT * n;
    // Lanes behind the last column load the first ones; what they sum is not stored.  A pair whose first column is the last one
    // begins one before it: the second sum is that column's.  Bytes from the step's first row on:
    const uint32_t at_code = 8u * half * a.ldq + (cm < ((a.F + 15) & ~15) ? cm : 0);
    const uint32_t at_g = 4u * (8u * half * a.ldg + (cn + NT <= a.H ? cn : NT == 2 && cn < a.H ? a.H - 2 : 0));

    f32x16 acc[MT][NT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int s = 0; s < NT; ++s)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[t][s][j] = 0.0f;

    // Addresses: those of the wave's rows, in scalar registers, and the lane's 32-bit offset.
    auto load = [&](GradRows<NT>& q, int64_t r0) {
        const char* code = reinterpret_cast<const char*>(a.codes) + r0 * a.ldq;
        const char* g = reinterpret_cast<const char*>(a.G) + r0 * a.ldg * 4;
#pragma unroll
        for (int j = 0; j < 2; ++j) q.scale[j] = *reinterpret_cast<const float4_u4*>(a.scale + r0 + 4 * j + 8u * half);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            q.code[j] = *reinterpret_cast<const typename GradCodes<MT>::type*>(code + (int64_t)j * a.ldq + at_code);
            const auto v = *reinterpret_cast<const typename GradPair<NT>::type*>(g + (int64_t)j * a.ldg * 4 + at_g);
#pragma unroll
            for (int s = 0; s < NT; ++s) q.g[j][s] = v[s];
        }
    };
    auto load_end = [&](GradRows<NT>& q, int64_t r0) {             // fewer than 16 rows: zeros behind them
        const int left = (int)(hi - r0) - 8 * half;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            q.code[j] = 0u;
            q.scale[j / 4][j % 4] = 0.0f;
#pragma unroll
            for (int s = 0; s < NT; ++s) q.g[j][s] = 0.0f;
            if (j < left) {
                const int64_t r = r0 + 8 * half + j;
                q.code[j] = *reinterpret_cast<const typename GradCodes<MT>::type*>(a.codes + (r0 + j) * a.ldq + at_code);
                q.scale[j / 4][j % 4] = a.scale[r];
                const float* p = reinterpret_cast<const float*>(reinterpret_cast<const char*>(a.G + (r0 + j) * a.ldg) + at_g);
#pragma unroll
                for (int s = 0; s < NT; ++s) q.g[j][s] = p[s];
            }
        }
    };
    auto multiply = [&](GradRows<NT>& q) {
        // what is loaded is first looked at here: the conversions stay behind the next step's loads
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            asm volatile("" : "+v"(q.code[j]), "+v"(q.scale[j / 4][j % 4]));
#pragma unroll
            for (int s = 0; s < NT; ++s) asm volatile("" : "+v"(q.g[j][s]));
        }
        GradFrag x[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < 8; j += 2)
                x[t].w[j / 2] = upper_halves((float)(int8_t)(q.code[j] >> (8 * t)), (float)(int8_t)(q.code[j + 1] >> (8 * t)));
#pragma unroll
        for (int s = 0; s < NT; ++s) {
            GradFrag y[3];
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                float v[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) v[u] = q.g[j + u][s] * q.scale[(j + u) / 4][(j + u) % 4];
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    y[p].w[j / 2] = upper_halves(v[0], v[1]);
#pragma unroll
                    for (int u = 0; u < 2; ++u) v[u] -= __uint_as_float(__float_as_uint(v[u]) & 0xFFFF0000u);
                }
            }
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[t][s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[t].v, y[p].v, acc[t][s], 0, 0, 0);
        }
    };

    GradRows<NT> q;
    const int64_t first = lo + wave * kGradStep, full = hi - first >= kGradStep ? (hi - first - kGradStep) / kGradRows + 1 : 0;
    if (full > 0) {
        load(q, first);
        for (int64_t s = 0; s < full; s += 2) {                // the next step's rows are requested before this one's are used
            GradRows<NT> next;
            load(next, first + min(s + 1, full - 1) * kGradRows);
            multiply(q);
            load(q, first + min(s + 2, full - 1) * kGradRows);
            if (s + 1 < full) multiply(next);
        }
    }
    if (first + full * kGradRows < hi) {
        load_end(q, first + full * kGradRows);
        multiply(q);
    }

    // ((wave 0 + wave 2) + (wave 1 + wave 3))
#pragma unroll
    for (int round = 2; round >= 1; --round) {
        if (wave >= round && wave < 2 * round) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int s = 0; s < NT; ++s)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sums[wave - round][((t * NT + s) * 16 + j) * kWaveSize + lane] = acc[t][s][j];
        }
        __syncthreads();
        if (wave < round) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int s = 0; s < NT; ++s)
#pragma unroll
                    for (int j = 0; j < 16; ++j) acc[t][s][j] += sums[wave][((t * NT + s) * 16 + j) * kWaveSize + lane];
        }
        __syncthreads();
    }
    if (wave > 0) return;
    float* out = a.dW + part * ((int64_t)a.F * a.ldw);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int32_t f = m0 + MT * (8 * (j / 4) + 4 * half + j % 4) + t;
            if (f >= a.F) continue;
            float* p = out + (int64_t)f * a.ldw + cn;
            if (cn + NT <= a.H) {
                typename GradPair<NT>::type v;
#pragma unroll
                for (int s = 0; s < NT; ++s) v[s] = acc[t][s][j];
                *reinterpret_cast<typename GradPair<NT>::type*>(p) = v;
            } else if (cn < a.H) {
                p[0] = acc[t][NT - 1][j];
            }
        }
}

constexpr int kGradJoin = 16;                                  // waves that share 64 elements of dW

// dW = the sum of the parts: wave w adds parts w, w + 16, ..., eight of which are requested at a time, and the waves' sums are
// added in their order.
__global__ void __launch_bounds__(kGradJoin * kWaveSize)
es_q8_grad_join_kernel(const float* __restrict__ part, int parts, int32_t F, int32_t H, float* __restrict__ dW, int32_t ldw)
{
    __shared__ float sums[kGradJoin][kWaveSize];
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    const int64_t size = (int64_t)F * H, i = (int64_t)blockIdx.x * kWaveSize + lane, at = min(i, size - 1);
    float s = 0.0f;
    for (int p = wave; p < parts; p += 8 * kGradJoin) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = part[min(p + u * kGradJoin, parts - 1) * size + at];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += p + u * kGradJoin < parts ? v[u] : 0.0f;
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave > 0 || i >= size) return;
    for (int w = 1; w < kGradJoin; ++w) s += sums[w][lane];
    dW[i / H * ldw + i % H] = s;
}

}  // namespace

#endif  // ES_SPMM_Q8_GRAD_H
