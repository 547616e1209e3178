// es_q8_spmm.h -- the sampled product on 8-bit rows, and the gradient of its entries' values.
//
//   Y[i, :]  = f_r * sum over the kept entries p of row r = rows[i] of  a_p * scale[c_p] * code[c_p, :]
//   dvals[p] = f_r * scale[c_p] * (dY[r, :] . code[c_p, :])  for a kept entry, 0 for the others
#ifndef ES_SPMM_Q8_SPMM_H
#define ES_SPMM_Q8_SPMM_H

#include "es_lanes.h"
#include "es_tile.h"

namespace {

constexpr int kQ8Cols = 16;                                    // columns a lane covers: one 128-bit load of codes
constexpr int kQ8Tile = 256;                                   // staged entries per wave

struct Q8Args {
    const int32_t* rowptr;
    const int32_t* colidx;
    const float* vals;
    const int8_t* codes;
    const float* scale;
    const int32_t* rows;
    float* Y;                  // the product, or (edge gradient) dvals
    const float* dY;
    float* partial;            // sums of parts of rows
    int64_t N, n_rows;
    uint64_t seed;
    int32_t F, ldq, ldy, W, mode, norm;
    uint32_t row_units;        // ldq / 16, the row stride of the codes in lane loads
    int32_t splits;            // parts a row may be cut into (few rows)
};

typedef uint32_t uint4_v __attribute__((ext_vector_type(4)));

// acc += w * the 16 codes of q
__device__ __forceinline__ void q8_fma(float (&acc)[kQ8Cols], float w, const uint4_v& q)
{
#pragma unroll
    for (int j = 0; j < kQ8Cols; ++j) acc[j] = fmaf(w, (float)(int8_t)(q[j / 4] >> (8 * (j % 4))), acc[j]);
}

// A row of the product: which row of the graph, and what is kept of it.
struct Q8Row {
    int64_t r;
    int32_t base, n, k;
};

__device__ __forceinline__ Q8Row q8_row(const Q8Args& a, int64_t i)
{
    Q8Row w = {-1, 0, 0, 0};
    if (i < a.n_rows) w.r = a.rows ? a.rows[i] : i;
    if (w.r < 0 || w.r >= a.N) w.r = -1;
    if (w.r >= 0) {
        w.base = a.rowptr[w.r];
        w.n = a.rowptr[w.r + 1] - w.base;
        w.k = kept_count(a.mode, w.n, a.W);
    }
    return w;
}

// Slots [t0, t0 + count) of a row into the tile, lane t of a team of `team`: the codes' place and the weight a_p * scale.
__device__ __forceinline__ void q8_stage(const Q8Args& a, RowSampler& s, int t, int team, int count, int32_t base, uint2* tile)
{
    sample_tile(s, t, team, count, [&](int slot, uint32_t entry) {
        const int64_t p = (int64_t)base + entry;
        const int32_t c = a.colidx[p];
        float w = a.scale[c];
        if (a.vals) w *= a.vals[p];
        tile[slot] = make_uint2((uint32_t)c, __float_as_uint(w));
    });
}

// The staged entries e, e + E, ... < count times their rows' 16 columns from `codes` (this lane's chunk) on.
template <int U>
__device__ __forceinline__ void q8_consume(const Q8Args& a, const uint2* tile, int count, int e, int E, const int8_t* codes,
                                           float (&acc)[kQ8Cols])
{
    for (int j = e; j < count; j += U * E) {
        uint2 ed[U];
        uint4_v q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int jj = j + u * E;
            ed[u] = tile[jj < count ? jj : j];
            if (jj >= count) ed[u].y = 0u;                     // codes are finite: weight 0 adds nothing
        }
#pragma unroll
        for (int u = 0; u < U; ++u) q[u] = *reinterpret_cast<const uint4_v*>(codes + (int64_t)ed[u].x * a.ldq);
#pragma unroll
        for (int u = 0; u < U; ++u) q8_fma(acc, __uint_as_float(ed[u].y), q[u]);
    }
}

// One wave per row, G lanes across 16 * G columns (blockIdx.y selects them), 64 / G entries side by side.
template <int G>
__global__ void __launch_bounds__(kBlockThreads) es_q8_spmm_kernel(const Q8Args a)
{
    constexpr int E = kWaveSize / G;
    __shared__ uint2 lds[kWavesPerBlock * kQ8Tile];
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    uint2* tile = lds + wave * kQ8Tile;
    const int64_t i = (int64_t)blockIdx.x * kWavesPerBlock + wave;
    const Q8Row w = q8_row(a, i);
    const int e = lane / G, l = lane % G;
    const int c0 = (blockIdx.y * G + l) * kQ8Cols;
    const int8_t* codes = a.codes + (c0 < a.F ? c0 : 0);
    RowSampler s;
    s.init(a.mode, a.seed, w.r, (uint32_t)w.n, (uint32_t)a.W, (uint32_t)lane, kWaveSize);
    float acc[kQ8Cols] = {};
    for (int t0 = 0; t0 < w.k; t0 += kQ8Tile) {
        const int count = min(w.k - t0, kQ8Tile);
        q8_stage(a, s, lane, kWaveSize, count, w.base, tile);
        wave_lds_fence();
        q8_consume<4>(a, tile, count, e, E, codes, acc);
        wave_lds_fence();
    }
#pragma unroll
    for (int j = 0; j < kQ8Cols; ++j)
        for (int m = G; m < kWaveSize; m <<= 1) acc[j] += __shfl_xor(acc[j], m, kWaveSize);
    if (i < a.n_rows && e == 0) {
        const float f = row_factor(a.norm, w.n, w.k);
        float* y = a.Y + i * (int64_t)a.ldy + c0;
#pragma unroll
        for (int j = 0; j < kQ8Cols; ++j)
            if (c0 + j < a.F) y[j] = acc[j] * f;
    }
}

// One wave per row; the lanes' shares of a dot product meet in registers.  Wider rows than 16 * G columns take
// several sweeps over the tile, whose sums meet in the tile.
template <int G>
__global__ void __launch_bounds__(kBlockThreads) es_q8_vals_kernel(const Q8Args a)
{
    constexpr int E = kWaveSize / G;
    __shared__ uint2 lds[kWavesPerBlock * kQ8Tile];
    __shared__ float sums[kWavesPerBlock * kQ8Tile];
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    uint2* tile = lds + wave * kQ8Tile;
    float* sum = sums + wave * kQ8Tile;
    const int64_t i = (int64_t)blockIdx.x * kWavesPerBlock + wave;
    const Q8Row w = q8_row(a, i);
    if (w.n == 0) return;
    const int e = lane / G, l = lane % G;
    const float f = row_factor(a.norm, w.n, w.k);
    float* out = a.Y + w.base;
    if (w.k < w.n) {
        const int from = a.mode == ES_BUCKET ? w.k : 0;
        for (int p = from + lane; p < w.n; p += kWaveSize) out[p] = 0.0f;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    }
    RowSampler s;
    s.init(a.mode, a.seed, w.r, (uint32_t)w.n, (uint32_t)a.W, (uint32_t)lane, kWaveSize);
    for (int t0 = 0; t0 < w.k; t0 += kQ8Tile) {
        const int count = min(w.k - t0, kQ8Tile);
        sample_tile(s, lane, kWaveSize, count, [&](int slot, uint32_t entry) {
            tile[slot] = make_uint2((uint32_t)a.colidx[(int64_t)w.base + entry], entry);
        });
        wave_lds_fence();
        for (int c = l * kQ8Cols; c - l * kQ8Cols < a.F; c += G * kQ8Cols) {
            float dy[kQ8Cols];
#pragma unroll
            for (int j = 0; j < kQ8Cols; ++j) dy[j] = c + j < a.F ? a.dY[w.r * (int64_t)a.ldy + c + j] : 0.0f;
            const int8_t* codes = a.codes + (c < a.F ? c : 0);
            for (int j0 = 0; j0 < count; j0 += E) {
                const int j = j0 + e;
                float d = 0.0f;
                if (j < count) {
                    const uint4_v q = *reinterpret_cast<const uint4_v*>(codes + (int64_t)tile[j].x * a.ldq);
#pragma unroll
                    for (int m = 0; m < kQ8Cols; ++m) d = fmaf(dy[m], (float)(int8_t)(q[m / 4] >> (8 * (m % 4))), d);
                }
                d = team_reduce<G>(d, [](float x, float y) { return x + y; });
                if (l == 0 && j < count) sum[j] = c == l * kQ8Cols ? d : sum[j] + d;
            }
        }
        wave_lds_fence();
        for (int j = lane; j < count; j += kWaveSize)
            out[tile[j].y] = sum[j] * (a.scale[tile[j].x] * f);
        wave_lds_fence();
    }
}

}  // namespace

#endif  // ES_SPMM_Q8_SPMM_H
