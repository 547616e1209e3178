// es_q8_spmm.h -- the sampled product on 8-bit rows, and the gradient of its entries' values.
//
//   Y[i, :]  = f_r * sum over the kept entries p of row r = rows[i] of  a_p * scale[c_p] * code[c_p, :]
//   dvals[p] = f_r * scale[c_p] * (dY[r, :] . code[c_p, :])  for a kept entry, 0 for the others
//
// A lane covers 16 columns, one 128-bit load of codes, and turns them into fp32 with one conversion and
// one fused multiply-add each; a whole line of 128 codes is gathered by 8 lanes.  G lanes cover a row's
// columns (blockIdx.y: which ones), R rows share a wave and E = 64 / (R G) entries of a row run side by side.  The weight
// a_p * scale[c_p] is formed where the entries are staged, one gather for 64 of them.
#ifndef ES_SPMM_Q8_SPMM_H
#define ES_SPMM_Q8_SPMM_H

#include "es_lanes.h"
#include "es_tile.h"

namespace {

constexpr int kQ8Cols = 16;                                    // columns of a lane
constexpr int kQ8Tile = 256;                                   // staged entries per wave
constexpr int kQ8TileStride = kQ8Tile + 64;                    // and pad slots between the rows' shares
constexpr int kQ8Batch = 4;                                    // loads of codes in flight per lane
constexpr int kQ8ScanRows = 1024;                              // rows that a group of long-row workgroups scans
constexpr int kQ8Share = 16;                                   // workgroups of such a group
static_assert(kQ8Share % kNumXcd == 0, "long-row workgroups must not shift the XCD phase");

struct Q8Args {
    const int32_t* rowptr;
    const int32_t* colidx;
    const float* vals;
    const int8_t* codes;
    const float* scale;
    const int32_t* rows;
    float* Y;                  // the product, or (edge gradient) dvals
    const float* dY;
    float* partial;            // sums of pieces of rows, F each
    int64_t N, n_rows;
    uint64_t seed;
    int32_t F, ldq, ldy, W, mode, norm;
    uint32_t row_units;        // ldq / 16: the row stride of the codes in lane loads
    int32_t long_k;            // rows keeping more entries are a workgroup's, not a wave's
    int32_t piece;             // and those keeping more than this are cut into pieces
    int64_t pieces;            // capacity of `partial`
    uint32_t nblocks, blocks_per_xcd, long_blocks;
    int32_t splits;            // es_q8_few_kernel: pieces a row may be cut into
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

// Where a column's codes are: a 32-bit count of lane loads where the whole table fits that (64 GiB), else the column itself.
template <bool WIDE>
__device__ __forceinline__ uint32_t q8_key(const Q8Args& a, int32_t c) { return WIDE ? (uint32_t)c : (uint32_t)c * a.row_units; }

template <bool WIDE>
__device__ __forceinline__ uint4_v q8_load(const Q8Args& a, const int8_t* codes, uint32_t key)
{
    const size_t at = WIDE ? (size_t)key * (size_t)a.ldq : (size_t)key * kQ8Cols;
    return *reinterpret_cast<const uint4_v*>(codes + at);
}

// Slots [0, count) of a tile, lane t of a team of `team`: the codes' place and the weight a_p * scale.
template <bool WIDE>
__device__ __forceinline__ void q8_stage(const Q8Args& a, RowSampler& s, int t, int team, int count, int32_t base, uint2* tile)
{
    sample_tile(s, t, team, count, [&](int slot, uint32_t entry) {
        const int64_t p = (int64_t)base + entry;
        const int32_t c = a.colidx[p];
        float w = a.scale[c];
        if (a.vals) w *= a.vals[p];
        tile[slot] = make_uint2(q8_key<WIDE>(a, c), __float_as_uint(w));
    });
}

// U entries from slot j on, E apart; those from `count` on add nothing: their weight is 0, and codes are finite.
template <int U, bool WIDE>
__device__ __forceinline__ void q8_batch(const Q8Args& a, const uint2* tile, int j, int count, int E, const int8_t* codes,
                                         float (&acc)[kQ8Cols])
{
    uint2 ed[U];
    uint4_v q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int jj = j + u * E;
        ed[u] = tile[jj < count ? jj : j];
        if (jj >= count) ed[u].y = 0u;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) q[u] = q8_load<WIDE>(a, codes, ed[u].x);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        q8_fma(acc, __uint_as_float(ed[u].y), q[u]);
        __builtin_amdgcn_sched_barrier(0);                     // or every load's codes are converted at once, into registers that spill
    }
}

// The staged entries e, e + E, ... < count.  The last batch is the smallest that holds every lane's rest.
template <bool WIDE>
__device__ __forceinline__ void q8_consume(const Q8Args& a, const uint2* tile, int count, int e, int E, const int8_t* codes,
                                           float (&acc)[kQ8Cols])
{
    constexpr int U = kQ8Batch;
    for (int j = e; j < count; j += U * E) {
        if (__ballot(j + U / 2 * E < count)) q8_batch<U, WIDE>(a, tile, j, count, E, codes, acc);
        else if (__ballot(j + E < count)) q8_batch<U / 2, WIDE>(a, tile, j, count, E, codes, acc);
        else q8_batch<1, WIDE>(a, tile, j, count, E, codes, acc);
    }
}

// Sums the lanes that are G, 2 G, ... apart inside a team.  Across the halves of a wave and the pairs of its
// rows of 16 lanes a register swap leaves each side half of the columns, so that what is left to sum
// halves each time; inside 16 lanes rotations add the rest.  Afterwards acc[0 .. COLS) are this lane's columns from `first` on.
template <int G, int TEAM>
struct Q8Sum {
    static constexpr int COLS = TEAM == 64 && G <= 16 ? 4 : TEAM == 32 && G <= 16 ? 8 : 16;
    static_assert(G <= 16 && TEAM >= 16, "a chunk of columns lies inside 16 lanes");
    __device__ __forceinline__ static int first(int lane)
    {
        return TEAM == 64 ? (lane >> 5) * 8 + (lane >> 4 & 1) * 4 : TEAM == 32 ? (lane >> 4 & 1) * 8 : 0;
    }
    __device__ __forceinline__ static void run(float (&acc)[kQ8Cols])
    {
        if constexpr (TEAM == 64) {
#pragma unroll
            for (int j = 0; j < 8; ++j) { lane_swap<false>(acc[j], acc[j + 8]); acc[j] += acc[j + 8]; }
        }
        if constexpr (TEAM >= 32) {
            constexpr int H = TEAM == 64 ? 4 : 8;
#pragma unroll
            for (int j = 0; j < H; ++j) { lane_swap<true>(acc[j], acc[j + H]); acc[j] += acc[j + H]; }
        }
        if constexpr (G <= 8) {
#pragma unroll
            for (int j = 0; j < COLS; ++j) acc[j] += dpp_move<0x128>(acc[j]);      // row_ror:8
        }
        if constexpr (G <= 4) {
#pragma unroll
            for (int j = 0; j < COLS; ++j) acc[j] += dpp_move<0x124>(acc[j]);
        }
        if constexpr (G <= 2) {
#pragma unroll
            for (int j = 0; j < COLS; ++j) acc[j] += dpp_move<0x122>(acc[j]);
        }
        if constexpr (G <= 1) {
#pragma unroll
            for (int j = 0; j < COLS; ++j) acc[j] += dpp_move<0x121>(acc[j]);
        }
    }
};

// COLS columns from c on into a row of F fp32 at any alignment; what the product writes it does not read again.
template <int COLS>
__device__ __forceinline__ void q8_store(float* y, int c, int F, const float (&acc)[kQ8Cols], float f)
{
    typedef float float4_u __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int j = 0; j < COLS; j += 4) {
        if (c + j + 4 <= F) {
            float4_u v = {acc[j] * f, acc[j + 1] * f, acc[j + 2] * f, acc[j + 3] * f};
            __builtin_nontemporal_store(v, reinterpret_cast<float4_u*>(y + c + j));
        } else {
#pragma unroll
            for (int m = 0; m < 4; ++m)
                if (c + j + m < F) y[c + j + m] = acc[j + m] * f;
        }
    }
}

// A whole workgroup on `count` slots of a row from slot t0 on; its wave 0 has the sum (as Q8Sum leaves it for a
// team of 64).  Every wave takes its own tiles in turn; their sums meet in LDS, in the waves' order.
template <int G, bool WIDE>
__device__ __forceinline__ void q8_block_sum(const Q8Args& a, const Q8Row& w, int32_t t0, int32_t count, const int8_t* codes,
                                             uint2* lds, float (&acc)[kQ8Cols])
{
    constexpr int E = kWaveSize / G;
    using Sum = Q8Sum<G, kWaveSize>;
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    uint2* tile = lds + wave * kQ8TileStride;
#pragma unroll
    for (int j = 0; j < kQ8Cols; ++j) acc[j] = 0.0f;
    // short pieces are dealt in shares of a batch, so that all four waves have some
    const int step = count >= kWavesPerBlock * kQ8Tile ? kQ8Tile : max(E * kQ8Batch, 64);
    for (int32_t s = wave * step; s < count; s += kWavesPerBlock * step) {
        RowSampler sampler;
        sampler.init(a.mode, a.seed, w.r, (uint32_t)w.n, (uint32_t)a.W, (uint32_t)(t0 + s + lane), kWaveSize);
        const int m = min(count - s, step);
        q8_stage<WIDE>(a, sampler, lane, kWaveSize, m, w.base, tile);
        wave_lds_fence();
        q8_consume<WIDE>(a, tile, m, lane / G, E, codes, acc);
        wave_lds_fence();
    }
    Sum::run(acc);
    float* part = reinterpret_cast<float*>(lds + kWavesPerBlock * kQ8TileStride);
    __syncthreads();
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < Sum::COLS; ++j) part[((wave - 1) * Sum::COLS + j) * kWaveSize + lane] = acc[j];
    }
    __syncthreads();
    if (wave == 0) {
        for (int v = 0; v < kWavesPerBlock - 1; ++v)
#pragma unroll
            for (int j = 0; j < Sum::COLS; ++j) acc[j] += part[(v * Sum::COLS + j) * kWaveSize + lane];
    }
}
constexpr int kQ8Lds = kWavesPerBlock * kQ8TileStride + (kWavesPerBlock - 1) * 4 * kWaveSize / 2;   // tiles and the waves' sums

// Place of the piece of a cut row that begins at its slot t0.  Pieces end where the CSR position, base + slot, is a multiple
// of `piece`; a span of `piece` positions can hold the end of one cut row and the beginning of another.
__device__ __forceinline__ int64_t q8_piece(const Q8Args& a, const Q8Row& w, int32_t t0)
{
    return 2 * (((int64_t)w.base + t0) / a.piece) + (t0 == 0 ? 1 : 0);
}
__device__ __forceinline__ int32_t q8_pieces(const Q8Args& a, const Q8Row& w)
{
    if (w.k <= a.piece) return 1;
    return (int32_t)(((int64_t)w.base + w.k - 1) / a.piece - w.base / a.piece) + 1;
}

struct Q8Scan {
    int end[kQ8ScanRows];
    int wave_total[kWavesPerBlock];
};

// Numbers the pieces of the long rows among rows [first, first + 1024); returns how many there are.
__device__ __forceinline__ int q8_scan(const Q8Args& a, int64_t first, Q8Scan& sc)
{
    constexpr int M = kQ8ScanRows / kBlockThreads;
    const int tid = threadIdx.x, lane = tid & (kWaveSize - 1), wave = tid >> 6;
    int count[M], mine = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const Q8Row w = q8_row(a, first + tid * M + i);
        count[i] = w.k > a.long_k ? q8_pieces(a, w) : 0;
        mine += count[i];
    }
    if (__syncthreads_or(mine) == 0) return 0;
    int incl = mine;
#pragma unroll
    for (int d = 1; d < kWaveSize; d <<= 1) {
        const int up = __shfl_up(incl, d, kWaveSize);
        if (lane >= d) incl += up;
    }
    if (lane == kWaveSize - 1) sc.wave_total[wave] = incl;
    __syncthreads();
    int before = incl - mine;
    for (int v = 0; v < wave; ++v) before += sc.wave_total[v];
#pragma unroll
    for (int i = 0; i < M; ++i) {
        before += count[i];
        sc.end[tid * M + i] = before;
    }
    __syncthreads();
    return sc.end[kQ8ScanRows - 1];
}

// The row, and which of its pieces, that has number `task` in that count.
__device__ __forceinline__ int q8_find(const Q8Scan& sc, int task, int& piece)
{
    int lo = 0, hi = kQ8ScanRows - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sc.end[mid] > task) hi = mid; else lo = mid + 1;
    }
    piece = task - (lo ? sc.end[lo - 1] : 0);
    return lo;
}

// The slots of piece number `piece` of row w.
__device__ __forceinline__ void q8_piece_slots(const Q8Args& a, const Q8Row& w, int piece, int32_t& t0, int32_t& count)
{
    if (w.k <= a.piece) { t0 = 0; count = w.k; return; }
    const int64_t span = w.base / a.piece + piece;             // positions [span * piece, (span + 1) * piece)
    const int64_t lo = max((int64_t)w.base, span * a.piece), hi = min((int64_t)w.base + w.k, (span + 1) * a.piece);
    t0 = (int32_t)(lo - w.base);
    count = (int32_t)(hi - lo);
}

// The product.  The leading workgroups take the long rows, whose waves would run long after the rest of the
// launch: 16 of them share those among 1024 rows.  The rest take R rows per wave, each XCD a contiguous range of rows.
template <int G, int R, bool WIDE>
__global__ void __launch_bounds__(kBlockThreads, 6) es_q8_spmm_kernel(const Q8Args a)
{
    constexpr int TEAM = kWaveSize / R, E = TEAM / G, T = kQ8Tile / R;
    __shared__ uint2 lds[kQ8Lds];
    __shared__ Q8Scan scan;
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    const int l = lane & (G - 1);
    const int c0 = (blockIdx.y * G + l) * kQ8Cols;
    const int8_t* codes = a.codes + (c0 < a.F ? c0 : 0);       // lanes behind the last column load the first ones
    float acc[kQ8Cols];

    if (blockIdx.x < a.long_blocks) {
        const int64_t first = (int64_t)(blockIdx.x / kQ8Share) * kQ8ScanRows;
        const int total = q8_scan(a, first, scan);
        for (int task = (blockIdx.x + blockIdx.x / kQ8Share) % kQ8Share; task < total; task += kQ8Share) {
            int piece, t0, count;
            const int64_t i = first + q8_find(scan, task, piece);
            const Q8Row w = q8_row(a, i);
            q8_piece_slots(a, w, piece, t0, count);
            q8_block_sum<G, WIDE>(a, w, t0, count, codes, lds, acc);
            if (wave == 0 && (lane & 15) < G) {
                using Sum = Q8Sum<G, kWaveSize>;
                const int c = c0 + Sum::first(lane);
                if (w.k <= a.piece) {
                    q8_store<Sum::COLS>(a.Y + i * (int64_t)a.ldy, c, a.F, acc, row_factor(a.norm, w.n, w.k));
                } else {
                    const int64_t at = q8_piece(a, w, t0);
                    if (at < a.pieces) q8_store<Sum::COLS>(a.partial + at * a.F, c, a.F, acc, 1.0f);
                }
            }
            __syncthreads();
        }
        return;
    }
    const uint32_t b = blockIdx.x - a.long_blocks;
    const uint32_t vb = (b % kNumXcd) * a.blocks_per_xcd + b / kNumXcd;
    if (vb >= a.nblocks) return;

    const int rs = lane / TEAM, t = lane & (TEAM - 1), e = t / G;
    uint2* tile = lds + wave * kQ8TileStride + rs * (T + E);   // the rows' slots j .. j + E - 1 miss each other's banks
    const int64_t i = ((int64_t)vb * kWavesPerBlock + wave) * R + rs;
    const Q8Row w = q8_row(a, i);
    const bool is_long = w.k > a.long_k;
    const int k = is_long ? 0 : w.k;
    RowSampler s;
    s.init(a.mode, a.seed, w.r, (uint32_t)w.n, (uint32_t)a.W, (uint32_t)t, TEAM);
#pragma unroll
    for (int j = 0; j < kQ8Cols; ++j) acc[j] = 0.0f;
    for (int t0 = 0; t0 < k; t0 += T) {
        const int count = min(k - t0, T);
        q8_stage<WIDE>(a, s, t, TEAM, count, w.base, tile);
        wave_lds_fence();
        q8_consume<WIDE>(a, tile, count, e, E, codes, acc);
        wave_lds_fence();
    }
    using Sum = Q8Sum<G, TEAM>;
    Sum::run(acc);
    if (i < a.n_rows && !is_long && (t & 15) < G)
        q8_store<Sum::COLS>(a.Y + i * (int64_t)a.ldy, c0 + Sum::first(lane), a.F, acc, row_factor(a.norm, w.n, w.k));
}

// Rows that were cut: the sum of their pieces in order, times the factor.
__global__ void __launch_bounds__(kBlockThreads) es_q8_join_kernel(const Q8Args a)
{
    __shared__ int any[kQ8ScanRows];
    __shared__ int found;
    const int64_t first = (int64_t)blockIdx.x * kQ8ScanRows;
    if (threadIdx.x == 0) found = 0;
    __syncthreads();
    for (int m = threadIdx.x; m < kQ8ScanRows; m += kBlockThreads)
        if (q8_row(a, first + m).k > a.piece) any[atomicAdd(&found, 1)] = m;   // their order is of no consequence
    __syncthreads();
    for (int x = 0; x < found; ++x) {
        const int64_t i = first + any[x];
        const Q8Row w = q8_row(a, i);
        const float f = row_factor(a.norm, w.n, w.k);
        const int64_t span = w.base / a.piece;
        const int pieces = q8_pieces(a, w);
        for (int c = threadIdx.x; c < a.F; c += kBlockThreads) {
            float s = 0.0f;
            for (int p = 0; p < pieces; ++p) {
                const int64_t at = 2 * (span + p) + (p == 0 ? 1 : 0);
                if (at < a.pieces) s += a.partial[at * a.F + c];
            }
            a.Y[i * (int64_t)a.ldy + c] = s * f;
        }
    }
}

// A few asked rows: every one is cut into up to a.splits equal pieces of 128 slots and more, a workgroup each.
__device__ __forceinline__ int32_t q8_few_length(const Q8Args& a, int32_t k)
{
    const int32_t each = (k - 1) / a.splits + 1;
    return each <= 128 ? 128 : (each + 63) & ~63;
}

template <int G, bool WIDE>
__global__ void __launch_bounds__(kBlockThreads) es_q8_few_kernel(const Q8Args a)
{
    using Sum = Q8Sum<G, kWaveSize>;
    __shared__ uint2 lds[kQ8Lds];
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    const int c0 = (blockIdx.y * G + (lane & (G - 1))) * kQ8Cols;
    const int8_t* codes = a.codes + (c0 < a.F ? c0 : 0);
    const int64_t i = blockIdx.x % a.n_rows;                   // pieces of one row go to different XCDs' queues last
    const int piece = (int)(blockIdx.x / a.n_rows);
    const Q8Row w = q8_row(a, i);
    const int32_t length = w.k ? q8_few_length(a, w.k) : 0;
    const int64_t t0 = (int64_t)piece * length;
    if (t0 >= w.k && !(piece == 0 && w.k == 0)) return;
    float acc[kQ8Cols];
    q8_block_sum<G, WIDE>(a, w, (int32_t)t0, (int32_t)min((int64_t)length, w.k - t0), codes, lds, acc);
    if (wave == 0 && (lane & 15) < G) {
        const int c = c0 + Sum::first(lane);
        if (w.k <= length) q8_store<Sum::COLS>(a.Y + i * (int64_t)a.ldy, c, a.F, acc, row_factor(a.norm, w.n, w.k));
        else q8_store<Sum::COLS>(a.partial + (i * a.splits + piece) * a.F, c, a.F, acc, 1.0f);
    }
}

__global__ void __launch_bounds__(kBlockThreads) es_q8_few_join_kernel(const Q8Args a)
{
    const int64_t i = blockIdx.x;
    const Q8Row w = q8_row(a, i);
    const int32_t length = w.k ? q8_few_length(a, w.k) : 0;
    if (w.k <= length) return;
    const float f = row_factor(a.norm, w.n, w.k);
    const int pieces = (w.k - 1) / length + 1;
    for (int c = blockIdx.y * kBlockThreads + threadIdx.x; c < a.F; c += gridDim.y * kBlockThreads) {
        float s = 0.0f;
        for (int p = 0; p < pieces; ++p) s += a.partial[(i * a.splits + p) * a.F + c];
        a.Y[i * (int64_t)a.ldy + c] = s * f;
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
