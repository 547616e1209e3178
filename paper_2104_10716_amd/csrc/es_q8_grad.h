// es_q8_grad.h -- dW = X^T G with X held as 8-bit rows: the weight gradient of a dense layer from its input's checkpoint.
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
    int64_t part_rows;         // rows of X that one part sums
};

constexpr int kGradTile = 64;                                  // rows and columns of dW per workgroup
constexpr int kGradStep = 16;                                  // rows of X staged at a time

// A workgroup sums a 64 x 64 tile of dW over its part's rows, 4 x 4 elements per thread.
__global__ void __launch_bounds__(kBlockThreads) es_q8_grad_kernel(const Q8Grad a)
{
    __shared__ float xs[kGradStep][kGradTile], gs[kGradStep][kGradTile];
    const int tid = threadIdx.x;
    const int m0 = blockIdx.x * kGradTile, n0 = blockIdx.y * kGradTile;
    const int64_t lo = blockIdx.z * a.part_rows, hi = min(a.N, lo + a.part_rows);
    const int tm = (tid / 16) * 4, tn = (tid % 16) * 4;
    float acc[4][4] = {};
    for (int64_t r0 = lo; r0 < hi; r0 += kGradStep) {
        for (int q = tid; q < kGradStep * kGradTile; q += kBlockThreads) {
            const int i = q / kGradTile, c = q % kGradTile;
            const int64_t r = r0 + i;
            xs[i][c] = r < hi && m0 + c < a.F ? (float)a.codes[r * a.ldq + m0 + c] * a.scale[r] : 0.0f;
            gs[i][c] = r < hi && n0 + c < a.H ? a.G[r * a.ldg + n0 + c] : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kGradStep; ++i)
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[m][n] = fmaf(xs[i][tm + m], gs[i][tn + n], acc[m][n]);
        __syncthreads();
    }
    float* out = a.dW + blockIdx.z * ((int64_t)a.F * a.ldw);
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (m0 + tm + m < a.F && n0 + tn + n < a.H) out[(int64_t)(m0 + tm + m) * a.ldw + n0 + tn + n] = acc[m][n];
}

// dW = the sum of the parts, in their order.
__global__ void __launch_bounds__(kBlockThreads)
es_q8_grad_join_kernel(const float* __restrict__ part, int parts, int32_t F, int32_t H, float* __restrict__ dW, int32_t ldw)
{
    const int64_t i = (int64_t)blockIdx.x * kBlockThreads + threadIdx.x, size = (int64_t)F * H;
    if (i >= size) return;
    float s = 0.0f;
    for (int p = 0; p < parts; ++p) s += part[p * size + i];
    dW[i / H * ldw + i % H] = s;
}

}  // namespace

#endif  // ES_SPMM_Q8_GRAD_H
