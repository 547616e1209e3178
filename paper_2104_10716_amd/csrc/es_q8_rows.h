// es_q8_rows.h -- rows as int8 codes with one fp32 scale per row: writing them and reading them back.
//
//   scale = fp32(max|x| / 127),  code_c = x_c / scale to the nearest integer, ties to even
//
// Both directions move each byte once and are bound by memory: a write reads F elements and writes F16 + 4
// bytes per row (F16: F rounded up to 16), a read the reverse: 2.45 M fp32 rows of 128, write 304 us (5.3 TB/s), read 250 us
// (6.3 TB/s); 16 k bf16 rows of 602 at random ids, write 13 us beside 6 us of marks, 64 k read 22 us (5.4 TB/s).
#ifndef ES_SPMM_Q8_ROWS_H
#define ES_SPMM_Q8_ROWS_H

#include "es_lanes.h"

namespace {

// 16 bytes of a dense row at any alignment of the element's own size: V elements (one 128-bit access: the HSA ABI runs
// the memory pipeline in unaligned-access mode).
template <class T>
struct Dense {
    static constexpr int V = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));

    __device__ __forceinline__ static void load(const T* p, int left, float (&v)[V])
    {
        if (left >= V) {
            const type q = *reinterpret_cast<const type*>(p);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = (float)q[j];
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = j < left ? (float)p[j] : 0.0f;
        }
    }
    __device__ __forceinline__ static void store(T* p, int left, const float (&v)[V])
    {
        if (left >= V) {
            type q;
#pragma unroll
            for (int j = 0; j < V; ++j) q[j] = (T)v[j];        // to nearest, ties to even
            *reinterpret_cast<type*>(p) = q;
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (j < left) p[j] = (T)v[j];
        }
    }
};

// V codes
template <int V> struct Codes { typedef uint32_t type __attribute__((ext_vector_type(V / 4))); };

// Scale of a row whose largest magnitude has these bits (as integers, magnitudes order like their values, infinity and
// NaN above every number).  Below 127 * 2^-126 the scale would be subnormal: such a row is
// held as zeros.  A row with an infinity or a NaN gets the scale NaN, and reads back as NaN.
__device__ __forceinline__ float q8_scale(uint32_t bits)
{
    if (bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const float m = __uint_as_float(bits);
    return m < 127.0f * 1.17549435e-38f ? 0.0f : fminf(m / 127.0f, 0x1.0204060000000p+121f);   // 127 times the bound is finite
}

__device__ __forceinline__ float q8_inverse(float scale) { return scale > 0.0f ? 1.0f / scale : 0.0f; }

// The codes of v.  x * (1 / scale) is within 2e-5 of the quotient, so its nearest integer is the
// quotient's or, next to a border, a neighbour of it; the remainder x - r * scale is a multiple of the
// smaller of the operands' last places and below scale in size, so the fused multiply-add has it exactly,
// and it says whether r is right.
template <int V>
__device__ __forceinline__ typename Codes<V>::type q8_codes(const float (&v)[V], float scale, float inv)
{
    float r[V], e[V];
    float worst = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        r[j] = rintf(v[j] * inv);
        e[j] = 2.0f * fmaf(-r[j], scale, v[j]);
        worst = fmaxf(worst, fabsf(e[j]));
    }
    if (worst >= scale) {                                      // a border, or a row held as zeros
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float a = fabsf(e[j]);
            if (a > scale || (a == scale && ((int)r[j] & 1))) r[j] += copysignf(1.0f, e[j]);
        }
    }
    typename Codes<V>::type words;
#pragma unroll
    for (int w = 0; w < V / 4; ++w) {
        uint32_t word = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) word |= ((uint32_t)(int)r[4 * w + j] & 0xFFu) << (8 * j);
        words[w] = scale > 0.0f ? word : 0u;                   // zeros for scale 0 and NaN
    }
    return words;
}

enum { Q8_ALL = 0, Q8_SCANNED = 1, Q8_CLAIMED = 2 };           // how the table's rows are named

struct Q8Write {
    const void* X;
    const int32_t* rows;
    int8_t* codes;
    float* scale;
    int64_t n, N;
    int32_t F, ldx, ldq;
};

// Rows whose index among a call's ids is at most this can be marked in the place of their scale (see below).
constexpr int64_t kQ8Claims = (1 << 23) - 2;
// Up to so many ids per lane of a team the ids are scanned: one launch instead of three, whose time grows with their number.  Random
// ids, us scanned / marked: F = 8 fp32 (4 lanes), 64 ids 4.4 / 7.4, 256 7.8 / 7.6, 1024 17.5 / 8.2; F = 64 (16 lanes), 1024 7.0 / 8.1, 2048
// 10.7 / 8.1; F = 128 bf16 (16 lanes), 512 8.3 / 10.3, 1024 12.5 / 10.3; F = 602 fp32 (32 lanes), 2048 5.8 / 7.2.
constexpr int64_t kQ8Scan = 50;

// Which table rows the elements i0 .. i0 + UR - 1 of the call go to, or -1.  Of equal ids the last one is written:
// Q8_SCANNED looks through the ids behind each; Q8_CLAIMED finds i + 1 in place of the row's scale
// (es_q8_claim_kernel).  A scale is 0, NaN or at least 2^-126, none of which has the bits of such a mark, so a
// reader that comes after the row's writer is not misled.  The whole team agrees.
template <int MAP, int TEAM, int UR>
__device__ __forceinline__ void q8_targets(const Q8Write& a, int64_t i0, int t, int64_t (&row)[UR])
{
    int32_t id[UR];
    uint32_t later[UR];
#pragma unroll
    for (int u = 0; u < UR; ++u) {
        row[u] = i0 + u < a.n ? i0 + u : -1;
        if (MAP == Q8_ALL) continue;
        id[u] = i0 + u < a.n ? a.rows[i0 + u] : -1;
        if (id[u] < 0 || id[u] >= a.N) id[u] = -1;
        row[u] = id[u];
        later[u] = 0;
    }
    if constexpr (MAP == Q8_CLAIMED) {
#pragma unroll
        for (int u = 0; u < UR; ++u) {
            if (id[u] < 0) continue;
            const uint32_t mark = __hip_atomic_load(reinterpret_cast<const uint32_t*>(a.scale) + id[u], __ATOMIC_RELAXED,
                                                    __HIP_MEMORY_SCOPE_AGENT);
            if (mark != (uint32_t)(i0 + u + 1)) row[u] = -1;
        }
    }
    if constexpr (MAP == Q8_SCANNED) {
        const int n = (int)a.n, at = (int)min(i0, a.n);        // both small
#pragma unroll 4
        for (int j = at + 1 + t; j < n; j += TEAM) {
            const int32_t other = a.rows[j];
#pragma unroll
            for (int u = 0; u < UR; ++u) later[u] |= j > at + u && other == id[u];
        }
#pragma unroll
        for (int u = 0; u < UR; ++u)
            if (team_reduce<TEAM>(later[u], [](uint32_t x, uint32_t y) { return x | y; })) row[u] = -1;
    }
}

// A team of TEAM lanes holds UR rows in registers, K loads of each per lane.  More rows at a time keep more bytes in flight; the
// rows are requested before it is known where, or whether, they go.
template <class T, int TEAM, int K, int UR, int MAP>
__global__ void __launch_bounds__(kBlockThreads) es_q8_write_kernel(const Q8Write a)
{
    constexpr int V = Dense<T>::V;
    const int t = threadIdx.x & (TEAM - 1);
    const int64_t i0 = ((int64_t)blockIdx.x * (kBlockThreads / TEAM) + threadIdx.x / TEAM) * UR;
    const int f16 = (a.F + 15) & ~15;
    float v[UR][K][V];
    int64_t row[UR];
#pragma unroll
    for (int u = 0; u < UR; ++u) {
        const T* x = static_cast<const T*>(a.X) + min(i0 + u, a.n - 1) * (int64_t)a.ldx;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TEAM + t) * V;
            Dense<T>::load(x + c, a.F - c, v[u][k]);
        }
    }
    q8_targets<MAP, TEAM>(a, i0, t, row);
#pragma unroll
    for (int u = 0; u < UR; ++u) {
        uint32_t bits = 0;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) bits = max(bits, __float_as_uint(v[u][k][j]) & 0x7FFFFFFFu);
        bits = team_reduce<TEAM>(bits, [](uint32_t x, uint32_t y) { return max(x, y); });
        if (row[u] < 0) continue;
        const float scale = q8_scale(bits);
        const float inv = q8_inverse(scale);
        int8_t* out = a.codes + row[u] * (int64_t)a.ldq;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TEAM + t) * V;
            if (c < f16) *reinterpret_cast<typename Codes<V>::type*>(out + c) = q8_codes(v[u][k], scale, inv);
        }
        if (t == 0)
            __hip_atomic_store(reinterpret_cast<uint32_t*>(a.scale) + row[u], __float_as_uint(scale), __ATOMIC_RELAXED,
                               __HIP_MEMORY_SCOPE_AGENT);
    }
}

// Rows too wide for a wave's registers: a workgroup per row reads it twice, the second time from the caches.
template <class T, int MAP>
__global__ void __launch_bounds__(kBlockThreads) es_q8_write_wide_kernel(const Q8Write a)
{
    constexpr int V = Dense<T>::V;
    __shared__ uint32_t part[kWavesPerBlock];
    const int64_t i = blockIdx.x;
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    int64_t rows[1];
    q8_targets<MAP, kWaveSize>(a, i, lane, rows);
    const int64_t row = rows[0];
    // every wave has to know before one of them replaces the mark
    __syncthreads();
    if (row < 0) return;
    const T* x = static_cast<const T*>(a.X) + i * (int64_t)a.ldx;
    const int64_t f16 = ((int64_t)a.F + 15) & ~(int64_t)15;
    uint32_t bits = 0;
    float v[V];
    for (int64_t c = threadIdx.x * V; c < a.F; c += kBlockThreads * V) {
        Dense<T>::load(x + c, (int)min((int64_t)V, a.F - c), v);
#pragma unroll
        for (int j = 0; j < V; ++j) bits = max(bits, __float_as_uint(v[j]) & 0x7FFFFFFFu);
    }
    bits = team_reduce<kWaveSize>(bits, [](uint32_t p, uint32_t q) { return max(p, q); });
    if (lane == 0) part[wave] = bits;
    __syncthreads();
    for (int w = 0; w < kWavesPerBlock; ++w) bits = max(bits, part[w]);
    const float scale = q8_scale(bits);
    const float inv = q8_inverse(scale);
    int8_t* out = a.codes + row * (int64_t)a.ldq;
    for (int64_t c = threadIdx.x * V; c < f16; c += kBlockThreads * V) {
        Dense<T>::load(x + c, (int)max((int64_t)0, min((int64_t)V, a.F - c)), v);
        *reinterpret_cast<typename Codes<V>::type*>(out + c) = q8_codes(v, scale, inv);
    }
    if (threadIdx.x == 0)
        __hip_atomic_store(reinterpret_cast<uint32_t*>(a.scale) + row, __float_as_uint(scale), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
}

// CLAIM == false: the scales of the rows to be written become 0; true: then the largest i + 1 of the ids i that name the row.
template <bool CLAIM>
__global__ void __launch_bounds__(kBlockThreads) es_q8_claim_kernel(const Q8Write a)
{
    const int64_t i = (int64_t)blockIdx.x * kBlockThreads + threadIdx.x;
    if (i >= a.n) return;
    const int32_t row = a.rows[i];
    if (row < 0 || row >= a.N) return;
    uint32_t* mark = reinterpret_cast<uint32_t*>(a.scale) + row;
    if (CLAIM)
        __hip_atomic_fetch_max(mark, (uint32_t)(i + 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else
        __hip_atomic_store(mark, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

struct Q8Read {
    const int8_t* codes;
    const float* scale;
    const int32_t* rows;
    void* Y;
    int64_t n, N;
    int32_t F, ldq, ldy;
};

// 16 bytes of Y per lane and store: the stores are most of the bytes.  K loads of each of UR rows are in flight per lane.
template <class T, int TEAM, int K, int UR>
__global__ void __launch_bounds__(kBlockThreads) es_q8_read_kernel(const Q8Read a)
{
    constexpr int V = Dense<T>::V;
    const int t = threadIdx.x & (TEAM - 1);
    const int64_t i0 = ((int64_t)blockIdx.x * (kBlockThreads / TEAM) + threadIdx.x / TEAM) * UR;
    int64_t row[UR];
    float scale[UR];
#pragma unroll
    for (int u = 0; u < UR; ++u) {
        row[u] = i0 + u;
        if (a.rows && i0 + u < a.n) row[u] = a.rows[i0 + u];
        if (i0 + u >= a.n || row[u] < 0 || row[u] >= a.N) row[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < UR; ++u) scale[u] = row[u] < 0 ? 0.0f : a.scale[row[u]];
    for (int64_t c0 = t * V; c0 - t * V < a.F; c0 += K * TEAM * V) {
        typename Codes<V>::type q[UR][K];
#pragma unroll
        for (int u = 0; u < UR; ++u)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int64_t c = c0 + k * TEAM * V;
                q[u][k] = 0u;
                if (row[u] >= 0 && c < a.F)
                    q[u][k] = *reinterpret_cast<const typename Codes<V>::type*>(a.codes + row[u] * (int64_t)a.ldq + c);
            }
#pragma unroll
        for (int u = 0; u < UR; ++u) {
            if (i0 + u >= a.n) continue;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int64_t c = c0 + k * TEAM * V;
                if (c >= a.F) continue;
                float v[V];
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = scale[u] * (float)(int8_t)(q[u][k][j / 4] >> (8 * (j % 4)));
                Dense<T>::store(static_cast<T*>(a.Y) + (i0 + u) * (int64_t)a.ldy + c, (int)min((int64_t)V, a.F - c), v);
            }
        }
    }
}

}  // namespace

#endif  // ES_SPMM_Q8_ROWS_H
