// es_q8_spmm.h -- the sampled product on 8-bit rows, and the gradient of its entries' values.
//
//   Y[i, :]  = f_r * sum over the kept entries p of row r = rows[i] of  a_p * scale[c_p] * code[c_p, :]
//   dvals[p] = f_r * scale[c_p] * (dY[r, :] . code[c_p, :])  for a kept entry, 0 for the others
//
// A lane covers 16 columns, one 128-bit load of codes, and turns them into fp32 with one conversion and
// one fused multiply-add each; a whole line of 128 codes is gathered by 8 lanes.  G lanes cover a row's
// columns (blockIdx.y: which ones).  The weight a_p * scale[c_p] is formed where the entries are staged.
#ifndef ES_SPMM_Q8_SPMM_H
#define ES_SPMM_Q8_SPMM_H

#include "es_lanes.h"
#include "es_tile.h"

namespace {

constexpr int kQ8Cols = 16;                                    // columns of a lane
constexpr int kQ8Tile = 256;                                   // staged entries per wave
constexpr int kQ8Batch = 4;                                     // loads of codes in flight per lane
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
    int32_t piece;             // and those keeping more than this are cut into pieces (the product's is at least long_k)
    int64_t pieces;            // capacity of `partial`
    uint32_t nblocks, blocks_per_xcd, long_blocks;
    int32_t splits;            // es_q8_few_kernel: pieces a row may be cut into
    int32_t wave_rows;         // rows of a wave, a power of two up to 64
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

// One tile of a row: TEAM lanes stage up to 4 TEAM entries from slot t0 on and multiply the first `most` of them (wave-uniform;
// no row of the wave has more here) with their rows' columns from `codes` on.  Slots from `count` on add
// nothing: their weight is 0, codes are finite, and they name a row of the table, that of entry `spare`.  All of a lane's
// loads of one kind are in flight together.
template <int G, int TEAM, bool WIDE>
__device__ __forceinline__ void q8_tile(const Q8Args& a, RowSampler& s, int t, int count, int most, int32_t base, int32_t spare,
                                        uint2* tile, const int8_t* codes, float (&acc)[kQ8Cols])
{
    constexpr int E = TEAM / G, U = kQ8Batch < 4 * G ? kQ8Batch : 4 * G;
    int64_t p[4];
    int32_t c[4];
    float w[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const uint32_t entry = s.next();
        p[m] = t + m * TEAM < count ? (int64_t)base + entry : (int64_t)spare;
        c[m] = a.colidx[p[m]];
    }
    if (a.vals) {
#pragma unroll
        for (int m = 0; m < 4; ++m) w[m] = a.vals[p[m]];
    } else {
#pragma unroll
        for (int m = 0; m < 4; ++m) w[m] = 1.0f;
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        w[m] *= a.scale[c[m]];
        tile[t + m * TEAM] = make_uint2(q8_key<WIDE>(a, c[m]), t + m * TEAM < count ? __float_as_uint(w[m]) : 0u);
    }
    wave_lds_fence();

    // edge slot e has the entries j + e U .. j + e U + U - 1 of each step of U E
    const uint4_v* pair = reinterpret_cast<const uint4_v*>(tile) + (t / G) * (U / 2);
#pragma unroll 1
    for (int j = 0; j < most; j += U * E) {
        uint4_v q[U];
        float x[U];
#pragma unroll
        for (int u = 0; u < U; u += 2) {
            const uint4_v two = pair[(j + u) / 2];
            q[u] = q8_load<WIDE>(a, codes, two[0]);
            q[u + 1] = q8_load<WIDE>(a, codes, two[2]);
            x[u] = __uint_as_float(two[1]);
            x[u + 1] = __uint_as_float(two[3]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            q8_fma(acc, x[u], q[u]);
            __builtin_amdgcn_sched_barrier(0);                 // or every load's codes are converted at once, into registers that spill
        }
    }
    wave_lds_fence();
}

// Sums the lanes of a team that are G, 2 G, ... apart.  Across the halves of a wave and the pairs of its rows of 16 lanes a
// register swap leaves each side half of the columns, so that what is left to sum halves each time; inside 16 lanes
// rotations add the rest.  Afterwards acc[0 .. COLS) are this lane's columns from `first` on.
template <int G, int TEAM>
struct Q8Sum {
    static constexpr int COLS = TEAM == 64 ? 4 : TEAM == 32 ? 8 : 16;
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
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            if constexpr (G <= 8) acc[j] += dpp_move<0x128>(acc[j]);               // row_ror:8
            if constexpr (G <= 4) acc[j] += dpp_move<0x124>(acc[j]);
            if constexpr (G <= 2) acc[j] += dpp_move<0x122>(acc[j]);
            if constexpr (G <= 1) acc[j] += dpp_move<0x121>(acc[j]);
        }
    }
};

// Columns c .. c + 3 of a row of F fp32 at any alignment; what the product writes it does not read again.
__device__ __forceinline__ void q8_store(float* y, int c, int F, const float* v, float f)
{
    typedef float float4_u __attribute__((ext_vector_type(4), aligned(4)));
    if (c + 4 <= F) {
        float4_u x = {v[0] * f, v[1] * f, v[2] * f, v[3] * f};
        __builtin_nontemporal_store(x, reinterpret_cast<float4_u*>(y + c));
    } else {
#pragma unroll
        for (int m = 0; m < 4; ++m)
            if (c + m < F) y[c + m] = v[m] * f;
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
    uint2* tile = lds + wave * kQ8Tile;
#pragma unroll
    for (int j = 0; j < kQ8Cols; ++j) acc[j] = 0.0f;
    // short pieces are dealt in smaller shares, so that all four waves have some
    const int step = count >= kWavesPerBlock * kQ8Tile ? kQ8Tile : max(E * kQ8Batch, 64);
    // slots unsigned: the one behind the last may be beyond 2^31
    for (uint32_t s = wave * step; s < (uint32_t)count; s += kWavesPerBlock * step) {
        RowSampler sampler;
        sampler.init(a.mode, a.seed, w.r, (uint32_t)w.n, (uint32_t)a.W, (uint32_t)t0 + s + lane, kWaveSize);
        const int m = (int)min((uint32_t)count - s, (uint32_t)step);
        q8_tile<G, kWaveSize, WIDE>(a, sampler, lane, m, m, w.base, w.base, tile, codes, acc);
    }
    Sum::run(acc);
    float* part = reinterpret_cast<float*>(lds + kWavesPerBlock * kQ8Tile);
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
constexpr int kQ8Lds = kWavesPerBlock * kQ8Tile + (kWavesPerBlock - 1) * 4 * kWaveSize / 2;   // tiles and the waves' sums

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

// What a wave keeps in LDS of each of its rows, in the order in which it takes them.
struct Q8Kept {
    int32_t base, n, k, place;                                 // place: among the wave's rows; -1: not this wave's to store
    uint32_t first, mult;                                      // FastRand: rotation and multiplier of a row that is sampled, else 0
};

// The rank of lane's k among those of the first `rows` lanes, largest first, ties by lane; the other lanes come behind them.
__device__ __forceinline__ int q8_rank(int k, int lane, int rows)
{
    int rank = 0;
    for (int j0 = 0; j0 < rows; j0 += 4)                       // lanes behind the rows have k = 0, and come behind any row
#pragma unroll
        for (int j = j0; j < j0 + 4; ++j) {
            const int other = __builtin_amdgcn_readlane(k, j);
            rank += (other > k || (other == k && j < lane)) ? 1 : 0;
        }
    return lane < rows ? rank : lane;
}

// The rows [first_row, first_row + wave_rows) of a wave: each lane works out one row, and the rows are put in the order of
// their kept entries, so that those that run side by side are of about one length.
__device__ __forceinline__ void q8_plan_rows(const Q8Args& a, int64_t first_row, int lane, Q8Kept* kept)
{
    Q8Row w = {-1, 0, 0, 0};
    if (lane < a.wave_rows) w = q8_row(a, first_row + lane);
    const bool mine = lane < a.wave_rows && first_row + lane < a.n_rows && w.k <= a.long_k;
    Q8Kept q = {w.base, w.n, mine ? w.k : 0, mine ? lane : -1, 0u, 0u};
    if (a.mode == ES_FASTRAND && q.k < w.n) {
        q.mult = fastrand_multiplier((uint32_t)w.n);
        q.first = fastrand_offset(a.seed, w.r, (uint32_t)w.n);
    }
    kept[q8_rank(q.k, lane, a.wave_rows)] = q;
    wave_lds_fence();
}

// Lane t of `team` on a row: the entries of slots t, t + team, ...
__device__ __forceinline__ void q8_sampler(RowSampler& s, const Q8Kept& w, int t, int team)
{
    s.idx = (uint32_t)t;
    s.step = (uint32_t)team;
    s.wrap = 0xFFFFFFFFu;
    if (w.mult) {
        s.idx = (w.first + (uint32_t)t * w.mult) % (uint32_t)w.n;
        s.step = ((uint32_t)team * w.mult) % (uint32_t)w.n;
        s.wrap = (uint32_t)w.n;
    }
}

// acc += the lanes of the team (of 4) that hold other entries of the same columns
template <int G, int TEAM>
__device__ __forceinline__ void q8_team_sum(float (&acc)[kQ8Cols])
{
    static_assert(TEAM == G || (TEAM == 4 && G < 4), "narrow rows: the quad's lanes");
#pragma unroll
    for (int j = 0; j < kQ8Cols; ++j) {
        if constexpr (TEAM > G && G <= 2) acc[j] += dpp_move<0x4E>(acc[j]);        // lanes two apart
        if constexpr (TEAM > G && G <= 1) acc[j] += dpp_move<0xB1>(acc[j]);        // and one apart
    }
}

// The product.  The leading workgroups take the long rows, whose waves would run long after the rest of the
// launch: 16 of them share those among 1024 rows.  The rest take wave_rows rows per wave, each XCD a contiguous range of
// rows: TEAM lanes to a row, 64 / TEAM rows side by side, TEAM / G entries of each at once.  TEAM is G, or 4, so that
// there is nothing, or little, to sum across lanes; or half a wave or a whole one, where rows are too few to fill the chip
// or long, and what counts is how soon the longest is done.
// An entry costs two requests to the L2, one line of codes and one of scales, or more where rows straddle lines, and a CU keeps
// some 100 of them in flight: that bounds the product (233 k rows, Bucket of 64, F = 64: 29.6 M requests of 384 clocks in 171 us, 1.0 GB
// behind the L2s; 2.45 M rows, FastRand of 64, F = 128: 120 M of 563 in 1300 us, 7.0 TB/s behind them; 170 k rows of mean 14, exact,
// F = 100: 6.7 M of 511 in 92 us).
// LONG: there may be long rows (a kernel of its own without them keeps its registers).
template <int G, int TEAM, bool LONG, bool WIDE>
__global__ void __launch_bounds__(kBlockThreads, 5) es_q8_spmm_kernel(const Q8Args a)
{
    constexpr int ROWS = kWaveSize / TEAM;
    constexpr int T = 4 * TEAM;                                // entries of a row staged at a time
    static_assert(T * ROWS == kQ8Tile, "");
    constexpr int ROW_SLOTS = T + 2;                           // and two of padding: the rows' entry j is in different banks
    constexpr int WAVE_SLOTS = ROWS * ROW_SLOTS > ROWS * G * kQ8Cols / 2 ? ROWS * ROW_SLOTS : ROWS * G * kQ8Cols / 2;
    constexpr int SLOTS = !LONG || kWavesPerBlock * WAVE_SLOTS > kQ8Lds ? kWavesPerBlock * WAVE_SLOTS : kQ8Lds;
    __shared__ __align__(16) uint2 lds[SLOTS];
    __shared__ union { Q8Kept kept[kWavesPerBlock][kWaveSize]; Q8Scan scan; } sh;
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    const int l = lane & (G - 1);
    const int c0 = (blockIdx.y * G + l) * kQ8Cols;
    const int8_t* codes = a.codes + min(c0, (a.F - 1) & -kQ8Cols);   // lanes behind the last columns load those: no line of their own
    float acc[kQ8Cols];

    if constexpr (LONG) {
        if (blockIdx.x < a.long_blocks) {
            const int64_t first = (int64_t)(blockIdx.x / kQ8Share) * kQ8ScanRows;
            const int total = q8_scan(a, first, sh.scan);
            for (int task = (blockIdx.x + blockIdx.x / kQ8Share) % kQ8Share; task < total; task += kQ8Share) {
                int piece, t0, count;
                const int64_t i = first + q8_find(sh.scan, task, piece);
                const Q8Row w = q8_row(a, i);
                q8_piece_slots(a, w, piece, t0, count);
                q8_block_sum<G, WIDE>(a, w, t0, count, codes, lds, acc);
                if (wave == 0 && (lane & 15) < G) {
                    const int c = c0 + Q8Sum<G, kWaveSize>::first(lane);
                    if (w.k <= a.piece) {
                        q8_store(a.Y + i * (int64_t)a.ldy, c, a.F, acc, row_factor(a.norm, w.n, w.k));
                    } else {
                        const int64_t at = q8_piece(a, w, t0);
                        if (at < a.pieces) q8_store(a.partial + at * a.F, c, a.F, acc, 1.0f);
                    }
                }
                __syncthreads();
            }
            return;
        }
    }
    const uint32_t b = blockIdx.x - a.long_blocks;
    const uint32_t vb = (b % kNumXcd) * a.blocks_per_xcd + b / kNumXcd;
    if (vb >= a.nblocks) return;

    const int64_t first_row = ((int64_t)vb * kWavesPerBlock + wave) * a.wave_rows;
    Q8Kept* kept = sh.kept[wave];
    q8_plan_rows(a, first_row, lane, kept);
    const int rs = lane / TEAM, t = lane & (TEAM - 1);
    uint2* own = lds + wave * WAVE_SLOTS;
    uint2* tile = own + rs * ROW_SLOTS;
    for (int p = rs; p < a.wave_rows; p += ROWS) {
        const Q8Kept w = kept[p];
        RowSampler s;
        q8_sampler(s, w, t, TEAM);
#pragma unroll
        for (int j = 0; j < kQ8Cols; ++j) acc[j] = 0.0f;
        // the first of the rows side by side keeps the most
        const int most = __builtin_amdgcn_readfirstlane(w.k), spare = __builtin_amdgcn_readfirstlane(w.base);
        for (int t0 = 0; t0 < most; t0 += T)
            q8_tile<G, TEAM, WIDE>(a, s, t, w.k - t0, min(most - t0, T), w.base, spare, tile, codes, acc);
        const float f = row_factor(a.norm, w.n, w.k);
        float* y = a.Y + (first_row + w.place) * (int64_t)a.ldy;
        if constexpr (TEAM > G && TEAM >= 16) {
            using Sum = Q8Sum<G, TEAM>;
            Sum::run(acc);
            if (w.place >= 0 && (lane & 15) < G) {
#pragma unroll
                for (int j = 0; j < Sum::COLS; j += 4) q8_store(y, c0 + Sum::first(lane) + j, a.F, acc + j, f);
            }
        } else {
            q8_team_sum<G, TEAM>(acc);
            // through LDS, so that a store instruction writes whole lines: lane t has the row's quads t, t + TEAM, ...
            float* out = reinterpret_cast<float*>(own) + rs * (G * kQ8Cols);
            if (t < G) {
#pragma unroll
                for (int j = 0; j < kQ8Cols; j += 4)
                    *reinterpret_cast<float4*>(out + l * kQ8Cols + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
            }
            wave_lds_fence();
#pragma unroll
            for (int q = 0; q < 4 * G; q += TEAM) {
                const float4 v = *reinterpret_cast<const float4*>(out + (q + t) * 4);
                const float v4[4] = {v.x, v.y, v.z, v.w};
                if (w.place >= 0) q8_store(y, blockIdx.y * G * kQ8Cols + (q + t) * 4, a.F, v4, f);
            }
            wave_lds_fence();
        }
    }
}

// The sum of `pieces` numbers in their order, eight of which are requested at a time.
template <class Get>
__device__ __forceinline__ float q8_sum_pieces(int pieces, Get&& get)
{
    float s = 0.0f;
    for (int p = 0; p < pieces; p += 8) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = get(min(p + u, pieces - 1));
#pragma unroll
        for (int u = 0; u < 8; ++u) s += p + u < pieces ? v[u] : 0.0f;
    }
    return s;
}

// Rows that were cut, which are all that keep more than `piece` entries: the sum of their pieces in order, times the factor.
__global__ void __launch_bounds__(kBlockThreads) es_q8_join_kernel(const Q8Args a)
{
    __shared__ int any[kQ8ScanRows];
    __shared__ int found;
    const int64_t first = (int64_t)blockIdx.x * kQ8ScanRows;
    if (threadIdx.x == 0) found = 0;
    __syncthreads();
    int32_t k[kQ8ScanRows / kBlockThreads];
#pragma unroll
    for (int m = 0; m < kQ8ScanRows / kBlockThreads; ++m) k[m] = q8_row(a, first + m * kBlockThreads + threadIdx.x).k;
#pragma unroll
    for (int m = 0; m < kQ8ScanRows / kBlockThreads; ++m)
        if (k[m] > a.piece) any[atomicAdd(&found, 1)] = m * kBlockThreads + threadIdx.x;   // their order is of no consequence
    __syncthreads();
    // a wave takes 64 columns of a row
    const int64_t groups = ((int64_t)a.F + kWaveSize - 1) / kWaveSize;
    for (int64_t task = threadIdx.x / kWaveSize; task < found * groups; task += kWavesPerBlock) {
        const int64_t i = first + any[task / groups], c = task % groups * kWaveSize + (threadIdx.x & (kWaveSize - 1));
        const Q8Row w = q8_row(a, i);
        const int64_t span = w.base / a.piece;
        if (c >= a.F) continue;
        const float s = q8_sum_pieces(q8_pieces(a, w), [&](int p) {
            const int64_t at = 2 * (span + p) + (p == 0 ? 1 : 0);
            return at < a.pieces ? a.partial[at * a.F + c] : 0.0f;
        });
        a.Y[i * (int64_t)a.ldy + c] = s * row_factor(a.norm, w.n, w.k);
    }
}

// A few asked rows: every one is cut into up to a.splits equal pieces of 128 slots and more, a workgroup each.  Latency bounds
// it: 32 rows of mean 490, F = 64: 4.3 us, and 2.8 us to join the pieces.
__device__ __forceinline__ int32_t q8_few_length(const Q8Args& a, int32_t k)
{
    if (a.splits == 1) return k;
    const int32_t each = (k - 1) / a.splits + 1;
    return each <= 128 ? 128 : (each + 63) & ~63;
}

template <int G, bool WIDE>
__global__ void __launch_bounds__(kBlockThreads) es_q8_few_kernel(const Q8Args a)
{
    using Sum = Q8Sum<G, kWaveSize>;
    __shared__ __align__(16) uint2 lds[kQ8Lds];               // read 16 bytes at a time
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    const int c0 = (blockIdx.y * G + (lane & (G - 1))) * kQ8Cols;
    const int8_t* codes = a.codes + min(c0, (a.F - 1) & -kQ8Cols);
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
        if (w.k <= length) q8_store(a.Y + i * (int64_t)a.ldy, c, a.F, acc, row_factor(a.norm, w.n, w.k));
        else q8_store(a.partial + (i * a.splits + piece) * a.F, c, a.F, acc, 1.0f);
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
        const float s = q8_sum_pieces(pieces, [&](int p) { return a.partial[(i * a.splits + p) * a.F + c]; });
        a.Y[i * (int64_t)a.ldy + c] = s * f;
    }
}

// ---- the gradient of the values ---------------------------------------------------------------
// This lane's 16 columns of a row of dY, from column c on; zeros behind the last one.
__device__ __forceinline__ void q8_load_dy(const Q8Args& a, int64_t r, int c, float (&dy)[kQ8Cols])
{
    typedef float float4_u __attribute__((ext_vector_type(4), aligned(4)));
    const float* p = a.dY + r * (int64_t)a.ldy + c;
#pragma unroll
    for (int j = 0; j < kQ8Cols; j += 4) {
        float4_u v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (c + j + 4 <= a.F) {
            v = *reinterpret_cast<const float4_u*>(p + j);
        } else {
#pragma unroll
            for (int m = 0; m < 4; ++m)
                if (c + j + m < a.F) v[m] = p[j + m];
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) dy[j + m] = v[m];
    }
}

// The first slot of lane t of a team, whose next ones are TEAM apart: the edge slots (G lanes each) have the first TEAM / G
// slots, then those behind them, so that a short row keeps all of them busy.
template <int G, int TEAM>
__device__ __forceinline__ int q8_slot(int t)
{
    return (t & (G - 1)) * (TEAM / G) + t / G;
}

// One tile of a row: TEAM lanes stage up to 4 TEAM entries, from slot `first` = q8_slot of the lane on; edge slot e then takes the
// entries of the lanes e G .. e G + G - 1, one after the other: G lanes multiply, their shares meet in registers, and the lane that
// staged an entry keeps its product.  `most`, `spare` as in q8_tile.  The gradients
// go to the entries' places, or by slot into `result` (LDS).  Rows wider than 16 G columns (G = 64) take several sweeps.
template <int G, int TEAM, bool WIDE>
__device__ __forceinline__ void q8_dots(const Q8Args& a, RowSampler& s, int t, int count, int most, int32_t base, int32_t spare,
                                        int64_t r, uint32_t* tile, float (&dy)[kQ8Cols], float f, float* result)
{
    constexpr int U = G < 4 ? G : 4, E = TEAM / G;
    const int l = t & (G - 1), e = t / G, first = q8_slot<G, TEAM>(t);
    int64_t p[4];
    int32_t c[4];
    float w[4], d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const uint32_t entry = s.next();
        p[m] = first + m * TEAM < count ? (int64_t)base + entry : (int64_t)spare;
        c[m] = a.colidx[p[m]];
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        w[m] = a.scale[c[m]] * f;
        tile[t + m * TEAM] = q8_key<WIDE>(a, c[m]);
    }
    wave_lds_fence();
    const uint32_t* key = tile + e * G;
    for (int c0 = l * kQ8Cols; c0 - l * kQ8Cols < a.F; c0 += G * kQ8Cols) {
        if constexpr (G == 64) q8_load_dy(a, r < 0 ? 0 : r, c0, dy);
        const int8_t* codes = a.codes + min(c0, (a.F - 1) & -kQ8Cols);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (m * TEAM >= most) break;                       // wave-uniform
#pragma unroll 1
            for (int u0 = 0; u0 < G; u0 += U) {
                if (m * TEAM + u0 * E >= most) break;
                uint4_v q[U];
#pragma unroll
                for (int u = 0; u < U; ++u) q[u] = q8_load<WIDE>(a, codes, key[m * TEAM + u0 + u]);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float x = 0.0f;
#pragma unroll
                    for (int j = 0; j < kQ8Cols; ++j) x = fmaf(dy[j], (float)(int8_t)(q[u][j / 4] >> (8 * (j % 4))), x);
                    x = team_reduce<G>(x, [](float y, float z) { return y + z; });
                    d[m] += l == u0 + u ? x : 0.0f;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        if (first + m * TEAM >= count) continue;
        if (result) result[first + m * TEAM] = d[m] * w[m];
        else a.Y[p[m]] = d[m] * w[m];
    }
    wave_lds_fence();
}

// dvals of entries [from, to), zeros; by `lanes` lanes
__device__ __forceinline__ void q8_zero(float* out, int64_t from, int64_t to, int lane, int lanes)
{
    typedef float float4_u __attribute__((ext_vector_type(4), aligned(4)));
    const float4_u zero = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t p = from + 4 * lane; p < to; p += 4 * lanes) {
        if (p + 4 <= to) {
            __builtin_nontemporal_store(zero, reinterpret_cast<float4_u*>(out + p));
        } else {
            for (int64_t q = p; q < to; ++q) out[q] = 0.0f;
        }
    }
}

// FastRand with W beyond what a wave can order in LDS: all gradients are cleared before any is written.
__global__ void __launch_bounds__(kBlockThreads) es_q8_zero_kernel(const Q8Args a)
{
    const int64_t from = a.rowptr[0], to = a.rowptr[a.N];
    q8_zero(a.Y, from, to, (int)(blockIdx.x * kBlockThreads + threadIdx.x), (int)(gridDim.x * kBlockThreads));
}

// Which slot of a FastRand row reads its entry 0, 1, ...: slot (idx - off) P^-1 mod n, Equation 2 solved for the slot.
struct Q8Slots {
    double inv_n;
    uint32_t slot0, step;                                      // entry 0's slot, and from one entry to the next
};

// (a * b) mod n for b < n < 2^31, a < 2^31, with 1 / n at hand
__device__ __forceinline__ uint32_t q8_mulmod(uint32_t a, uint32_t b, uint32_t n, double inv_n)
{
    const uint64_t q = (uint64_t)((double)a * (double)b * inv_n);          // off by one at most
    int64_t rem = (int64_t)((uint64_t)a * b - q * n);
    if (rem < 0) rem += n;
    if (rem >= (int64_t)n) rem -= n;
    return (uint32_t)rem;
}

__device__ __forceinline__ Q8Slots q8_slots(const Q8Kept& w)
{
    Q8Slots s = {1.0 / (double)max(w.n, 1), 0u, 1u};           // a row kept whole: entry idx is slot idx
    if (w.mult) {
        // With n = P a + r: P x = 1 + n m for m = -r^-1 mod P, so x = P^-1 mod n = a m + (1 + r m) / P.  P is a prime below
        // 600 that does not divide n.
        const uint32_t P = w.mult, n = (uint32_t)w.n, a = n / P, r = n % P;
        int32_t u = (int32_t)P, v = (int32_t)r, x0 = 0, x1 = 1;            // u = x0 r, v = x1 r (mod P)
        while (v > 1) {
            const int32_t q = u / v, next = u - q * v, x = x0 - q * x1;
            u = v; v = next; x0 = x1; x1 = x;
        }
        const uint32_t m = x1 < 0 ? (uint32_t)-x1 : P - (uint32_t)x1;
        s.step = a * m + (1u + r * m) / P;
        s.slot0 = w.first ? q8_mulmod(n - w.first, s.step, n, s.inv_n) : 0u;
    }
    return s;
}

constexpr int32_t kQ8MostRandom = 1024;                        // largest W whose gradients a wave orders in LDS

enum { Q8_PREFIX = 0, Q8_LONG = 1, Q8_RANDOM = 2 };

// Rows and waves as in es_q8_spmm_kernel, and the same bound, next to reading dY and writing dvals (170 k rows of mean 14, Bucket of 16,
// F = 128: 39 us, 5.8 TB/s; 233 k of mean 490, FastRand of 64, F = 41: 393 us, 36.9 M requests).  What is not kept gets its zeros in
// the same pass:
//  * Q8_PREFIX: all of a row is kept, or its first entries (full, Bucket); the wave clears what is behind them
//  * Q8_LONG: the same where there may be long rows; here and in Q8_PREFIX FastRand's zeros are there before (es_q8_zero_kernel)
//  * Q8_RANDOM: the kept entries lie anywhere in the row.  Zeros and gradients written one after the other would be two
//    writes of each line, the second of single numbers; instead the gradients stay in LDS by slot, and each
//    entry looks up whether a slot reads it, so that the row is written once, in order.
template <int G, int TEAM, int KIND, bool WIDE>
__global__ void __launch_bounds__(kBlockThreads, 4) es_q8_vals_kernel(const Q8Args a)
{
    constexpr int ROWS = kWaveSize / TEAM, T = 4 * TEAM;
    constexpr int RESULTS = KIND != Q8_RANDOM ? 1 : kQ8MostRandom / ROWS;   // kept entries of a row, at most
    __shared__ uint32_t lds[kWavesPerBlock * kQ8Tile];
    __shared__ float results[kWavesPerBlock * ROWS * RESULTS];
    __shared__ Q8Slots slots[KIND == Q8_RANDOM ? kWavesPerBlock * kWaveSize : 1];
    __shared__ union { Q8Kept kept[kWavesPerBlock][kWaveSize]; Q8Scan scan; } sh;
    const int lane = threadIdx.x & (kWaveSize - 1), wave = threadIdx.x >> 6;
    float dy[kQ8Cols];
    if constexpr (KIND == Q8_LONG) {
        if (blockIdx.x < a.long_blocks) {
            const int64_t first = (int64_t)(blockIdx.x / kQ8Share) * kQ8ScanRows;
            const int total = q8_scan(a, first, sh.scan);
            for (int task = (blockIdx.x + blockIdx.x / kQ8Share) % kQ8Share; task < total; task += kQ8Share) {
                int piece, t0, count;
                const Q8Row w = q8_row(a, first + q8_find(sh.scan, task, piece));
                q8_piece_slots(a, w, piece, t0, count);
                if (a.mode == ES_BUCKET && t0 == 0) q8_zero(a.Y, (int64_t)w.base + w.k, (int64_t)w.base + w.n, threadIdx.x, kBlockThreads);
                if constexpr (G < 64) q8_load_dy(a, w.r, (lane & (G - 1)) * kQ8Cols, dy);
                const float f = row_factor(a.norm, w.n, w.k);
                for (int s0 = wave * kWaveSize; s0 < count; s0 += kBlockThreads) {
                    RowSampler s;
                    s.init(a.mode, a.seed, w.r, (uint32_t)w.n, (uint32_t)a.W, (uint32_t)(t0 + s0 + q8_slot<G, kWaveSize>(lane)), kWaveSize);
                    const int m = min(count - s0, kWaveSize);
                    q8_dots<G, kWaveSize, WIDE>(a, s, lane, m, m, w.base, w.base, w.r, lds + wave * kQ8Tile, dy, f, nullptr);
                }
            }
            return;
        }
    }
    const uint32_t b = blockIdx.x - a.long_blocks;
    const uint32_t vb = (b % kNumXcd) * a.blocks_per_xcd + b / kNumXcd;
    if (vb >= a.nblocks) return;
    const int64_t first_row = ((int64_t)vb * kWavesPerBlock + wave) * a.wave_rows;
    Q8Kept* kept = sh.kept[wave];
    Q8Slots* slot = slots + (KIND == Q8_RANDOM ? wave * kWaveSize : 0);
    q8_plan_rows(a, first_row, lane, kept);
    if constexpr (KIND == Q8_RANDOM) {
        slot[lane] = q8_slots(kept[lane]);
        wave_lds_fence();
    }
    const int rs = lane / TEAM, t = lane & (TEAM - 1);
    uint32_t* tile = lds + wave * kQ8Tile + rs * T;
    float* result = results + wave * ROWS * RESULTS;
    for (int p0 = 0; p0 < a.wave_rows; p0 += ROWS) {
        const Q8Kept w = kept[p0 + rs];
        const int64_t r = w.place < 0 ? -1 : first_row + w.place;
        const int most = __builtin_amdgcn_readfirstlane(w.k), spare = __builtin_amdgcn_readfirstlane(w.base);
        if (most == 0) break;                                  // and so are all that follow
        RowSampler s;
        q8_sampler(s, w, q8_slot<G, TEAM>(t), TEAM);
        if constexpr (G < 64) q8_load_dy(a, r < 0 ? 0 : r, (t & (G - 1)) * kQ8Cols, dy);
        const float f = row_factor(a.norm, w.n, w.k);
        for (int t0 = 0; t0 < most; t0 += T)
            q8_dots<G, TEAM, WIDE>(a, s, t, w.k - t0, min(most - t0, T), w.base, spare, r, tile, dy, f,
                                   KIND == Q8_RANDOM ? result + rs * RESULTS + t0 : nullptr);
        if constexpr (KIND == Q8_RANDOM) {
            // the whole wave on one row after the other, four entries of it per lane
            for (int x = 0; x < ROWS; ++x) {
                const Q8Kept o = kept[p0 + x];
                const Q8Slots z = slot[p0 + x];
                const uint32_t n = (uint32_t)__builtin_amdgcn_readfirstlane(o.n), k = (uint32_t)__builtin_amdgcn_readfirstlane(o.k);
                if (k == 0) break;
                typedef float float4_u __attribute__((ext_vector_type(4), aligned(4)));
                const uint32_t jump = q8_mulmod(4 * kWaveSize, z.step, n, z.inv_n);
                uint32_t at = z.slot0 + q8_mulmod(4u * lane, z.step, n, z.inv_n);
                if (at >= n) at -= n;
                float* out = a.Y + o.base;
                for (uint32_t idx = 4u * lane; idx < n; idx += 4 * kWaveSize) {
                    float4_u v;
                    uint32_t i = at;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v[j] = i < k ? result[x * RESULTS + i] : 0.0f;
                        i += z.step;
                        if (i >= n) i -= n;
                    }
                    if (idx + 4 <= n) {
                        __builtin_nontemporal_store(v, reinterpret_cast<float4_u*>(out + idx));   // out of the codes' way in the L2
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (idx + j < n) out[idx + j] = v[j];
                    }
                    at += jump;
                    if (at >= n) at -= n;
                }
            }
            wave_lds_fence();
        }
    }
    if (KIND != Q8_RANDOM && a.mode == ES_BUCKET) {
        for (int x = 0; x < a.wave_rows; ++x) {
            const Q8Kept o = kept[x];
            if (o.place >= 0) q8_zero(a.Y, (int64_t)o.base + o.k, (int64_t)o.base + o.n, lane, kWaveSize);
        }
    }
}

}  // namespace

#endif  // ES_SPMM_Q8_SPMM_H
