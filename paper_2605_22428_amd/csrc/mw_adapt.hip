// mw_adapt, mw_adapt_backward: low-rank adapters of many requests beside a shared projection.
//
//   y_t  = base_t + c_a B_a h_t,   h_t = A_a x_t                       a: the adapter of row t
//   dh_t = B_a^T dy_t,   dx_t = dx_base_t + c_a A_a^T dh_t,   dA_a = c_a sum_t dh_t x_t^T,   dB_a = c_a sum_t dy_t h_t^T
//
// Rows are put in order of their adapters first (stable, so sums over an adapter's rows have one order) and cut into tiles of one
// adapter each.  k_adapt_down makes h of a tile, its workgroups sharing the columns of x out where there are few tiles; k_adapt_up adds
// up their parts and makes a slice of y.  The gradient of the input is the same walk with the transposed factors; beside it the
// tiles' h and dh are laid out for k_adapt_grads, which goes over an adapter's rows of x and dy once more.
//
// Forward each row of x, base and y is touched once, the factors come out of the caches: bytes bound large calls, launches and chains of round
// trips small ones.  Backward goes over x and dy again for every 32 ranks, out of the caches where they hold them, and is bound by that.  Measured
// on one MI355X: 8192 rows, 8 adapters of rank 32, 7168 to 4096 (246 MB): order 9 us, k_adapt_down 26 us (4.5 TB/s of x), k_adapt_up 31 us (4.3
// TB/s of base and y), the call 66 us.  64 rows of 24 adapters, rank 16, 7168 to 7168: 5.6 and 8.6 us, the call 13.5 us.  Backward of 4096 rows, 4
// adapters of rank 64, 4096 to 4096 (144 MB): prepare 7.5, down 16, up 30, k_adapt_grads 32.5 us (2.1 TB/s), the call 82 to 85 us.
#include "mw_stream.h"

namespace {

constexpr int kOrderBlock = 1024, kOrderWaves = kOrderBlock / 64;
constexpr int kBins = MW_ADAPT_MAX_ADAPTERS + 1;       // the last: rows without an adapter

struct adapt_tile { int32_t adapter, first, count, reserved0; };      // adapter == n_adapters: rows without one

struct order_args {
    const int32_t *ids;
    int32_t T, n, tile_rows, most_tiles;
    int32_t *order;                        // rows by (adapter, row)
    int32_t *tile_at;                      // [n + 2] first tile of an adapter, of the rows without one, and how many there are
    adapt_tile *tiles;
    uint32_t *flags;
};

// One workgroup.
__device__ __forceinline__ void make_order(const order_args &a, char *order_stage)
{
    extern __shared__ uint32_t order_lds[];                   // (by the adapters there are: the transposing workgroups are given it too)
    __shared__ uint32_t scratch[17];
    const int n_bins = a.n + 1;
    uint32_t *row_at = order_lds, *tile_at = row_at + n_bins + 1, *hists = tile_at + n_bins + 1;
    constexpr int kHeld = 8;               // pieces of 64 ids a wave requests together
    uint16_t (*held)[kHeld * 64] = (uint16_t (*)[kHeld * 64])order_stage, (*placed)[kHeld * 64] = held + kOrderWaves;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = a.n, T = a.T;
    const int per = ((T + kOrderWaves - 1) / kOrderWaves + 63) / 64 * 64;      // a wave's rows, in pieces of 64
    const int lo = wave * per, hi = min(T, lo + per);
    uint32_t *hist = hists + wave * n_bins;
    bool wrong = false;
    // Bins of the rows from `at`.  They wait in LDS for loops that are not unrolled: code that runs once is fetched at memory's pace.
    auto hold = [&](int at) {
        int id[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) id[i] = at + i * 64 + lane < hi ? a.ids[at + i * 64 + lane] : -1;
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            wrong |= id[i] < -1 || id[i] >= n;
            held[wave][i * 64 + lane] = (uint16_t)(id[i] < 0 || id[i] >= n ? n : id[i]);
        }
    };
    // The place of every row of the piece from t0 among the wave's rows of its adapter; hist counts them.  (64 lanes' atomics to one place are
    // one after the other for the whole workgroup: rows of few adapters took 13 us to count so, 8192 of them.)
    int bits = 0;
    while ((1 << bits) <= n) ++bits;
    auto place = [&](int t, int b) {
        const bool live = t < hi;
        unsigned long long same = __ballot(live);              // the piece's rows of the same adapter
        if (__ballot(live && b != __builtin_amdgcn_readfirstlane(b)) != 0)
            for (int i = 0; i < bits; ++i) {
                const unsigned long long set = __ballot((b >> i) & 1);
                same &= (b >> i) & 1 ? set : ~set;
            }
        const int before = __popcll(same & ((1ull << lane) - 1));
        const uint32_t at = hist[b] + (uint32_t)before;
        __builtin_amdgcn_wave_barrier();
        if (live && before == 0) hist[b] += (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
        return at;
    };
    for (int i = lane; i <= n; i += 64) hist[i] = 0;
    for (int at = lo; at < hi; at += kHeld * 64) {
        hold(at);
#pragma unroll 1
        for (int t0 = at; t0 < min(hi, at + kHeld * 64); t0 += 64) {
            const int i = t0 - at + lane;
            placed[wave][i] = (uint16_t)place(t0 + lane, held[wave][i]);
        }
    }
    if (a.flags && wrong) atomicOr(a.flags, MW_FLAG_BAD_ADAPTER);
    mw_lds_barrier();
    // places: bins in order, in a bin the waves in order
    constexpr int kPer = (kBins + kOrderBlock - 1) / kOrderBlock;
    uint32_t rows[kPer], rsum = 0, tsum = 0, total;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = tid * kPer + i;
        rows[i] = 0;
        if (b <= n)
            for (int w = 0; w < kOrderWaves; ++w) rows[i] += hists[w * n_bins + b];
        rsum += rows[i];
        tsum += (rows[i] + a.tile_rows - 1) / a.tile_rows;
    }
    uint32_t r = mw_block_exscan(rsum, scratch, &total);
    uint32_t k = mw_block_exscan(tsum, scratch, &total);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = tid * kPer + i;
        if (b <= n) {
            row_at[b] = r;
            tile_at[b] = k;
            a.tile_at[b] = (int32_t)k;
            uint32_t p = r;
            for (int w = 0; w < kOrderWaves; ++w) {
                const uint32_t c = hists[w * n_bins + b];
                hists[w * n_bins + b] = p;
                p += c;
            }
        }
        r += rows[i];
        k += (rows[i] + a.tile_rows - 1) / a.tile_rows;
    }
    if (tid == 0) {
        row_at[n + 1] = (uint32_t)T;
        tile_at[n + 1] = total;
        a.tile_at[n + 1] = (int32_t)total;
    }
    mw_lds_barrier();
    for (int i = (int)total + tid; i < a.most_tiles; i += kOrderBlock) a.tiles[i] = adapt_tile{-1, 0, 0, 0};
    for (int i = tid; i < (int)total; i += kOrderBlock) {      // the bin a tile is of: the last that starts at or before it
        int at = 0, end = n + 1;
        while (end - at > 1) {
            const int mid = (at + end) / 2;
            if (tile_at[mid] <= (uint32_t)i) at = mid; else end = mid;
        }
        const int first = (int)row_at[at] + (i - (int)tile_at[at]) * a.tile_rows;
        a.tiles[i] = adapt_tile{at, first, min(a.tile_rows, (int)row_at[at + 1] - first), 0};
    }
    if (hi - lo <= kHeld * 64) {           // the wave's rows and their places are still there
        for (int t = lo + lane; t < hi; t += 64) a.order[hist[held[wave][t - lo]] + placed[wave][t - lo]] = t;
        return;
    }
    for (int at = lo; at < hi; at += kHeld * 64) {
        hold(at);
#pragma unroll 1
        for (int t0 = at; t0 < min(hi, at + kHeld * 64); t0 += 64) {
            const uint32_t to = place(t0 + lane, held[wave][t0 - at + lane]);
            if (t0 + lane < hi) a.order[to] = t0 + lane;
        }
    }
}
constexpr int kStageBytes = 2 * kOrderWaves * 8 * 64 * 2;  // ids that wait, and their places
__global__ __launch_bounds__(kOrderBlock) void k_adapt_order(order_args a)
{
    __shared__ __align__(16) char stage[kStageBytes];
    make_order(a, stage);
}
uint32_t order_lds_bytes(int32_t n) { return (uint32_t)((n + 2) * 2 + (n + 1) * kOrderWaves) * 4; }

// The order in workgroup 0; the others transpose the factors: [n][rows][cols] -> [n][cols][rows], 64 x 128 values a piece.  As many workgroups
// as there are pieces, or kMostPieces, each then a piece every so many (a grid holds less than 2^32 threads: 1024 adapters of 262144 values have more).
struct transpose_args { const uint16_t *in; uint16_t *out; int32_t rows, cols; };
constexpr int64_t kMostPieces = 1 << 20;
__host__ __device__ __forceinline__ int64_t pieces_of(const transpose_args &t) { return (int64_t)((t.rows + 63) / 64) * ((t.cols + 127) / 128); }
__global__ __launch_bounds__(kOrderBlock) void k_adapt_prepare(order_args a, transpose_args t0, transpose_args t1)
{
    __shared__ __align__(16) char stage[kStageBytes];
    uint16_t (*tiles)[64][72] = (uint16_t (*)[64][72])stage;    // each half of the workgroup has its own
    static_assert(2 * 64 * 72 * 2 <= kStageBytes, "room for two of them");
    if (blockIdx.x == 0) {
        make_order(a, stage);
        return;
    }
    const int64_t per0 = pieces_of(t0), all = (per0 + pieces_of(t1)) * a.n;
    for (int64_t piece = (int64_t)blockIdx.x - 1; piece < all; piece += (int64_t)gridDim.x - 1) {
        const bool first = piece < per0 * a.n;
        const transpose_args t = first ? t0 : t1;
        const int64_t at = first ? piece : piece - per0 * a.n;
        const int64_t wide = (t.cols + 127) / 128, per = pieces_of(t), matrix = at / per;
        const int r0 = (int)(at % per / wide) * 64, c0 = (int)(at % wide) * 128 + (int)(threadIdx.x >> 9) * 64, i = threadIdx.x >> 3 & 63, q = (threadIdx.x & 7) * 8;
        const int64_t base = matrix * t.rows * t.cols;
        uint16_t (*tile)[72] = tiles[threadIdx.x >> 9];
        if (r0 + i < t.rows && c0 + q < t.cols) *(u32x4 *)&tile[i][q] = *(const u32x4 *)(t.in + base + (int64_t)(r0 + i) * t.cols + c0 + q);
        __syncthreads();
        if (c0 + i < t.cols && r0 + q < t.rows) {              // (rows and columns are multiples of 8)
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = tile[q + 2 * j][i] | (uint32_t)tile[q + 2 * j + 1][i] << 16;
            *(u32x4 *)(t.out + base + (int64_t)(c0 + i) * t.rows + r0 + q) = u32x4{v[0], v[1], v[2], v[3]};
        }
        __syncthreads();
    }
}

struct adapt_args {
    const int32_t *order; const adapt_tile *tiles;      // null: every workgroup finds its tile in the ids (at most kBlock rows)
    const int32_t *ids; uint32_t *flags;
    const uint16_t *a, *b;                 // [n][rank][n_in], [n][n_out][rank]
    const float *scale;                    // [n] or null
    int32_t T, n, rank, n_in, n_out;
    const uint16_t *x; int64_t x_stride;
    const uint16_t *base; int64_t base_stride;     // or null
    uint16_t *out; int64_t out_stride;
    int32_t slice, n_slices;               // columns of x a workgroup of k_adapt_down takes
    int32_t out_slice;                     // columns of y a workgroup of k_adapt_up takes
    float *part;                           // [n_slices][T][ranks, whole tiles]
    float *h;                              // [T][rank] or null
    // for k_adapt_grads, or null: c h and c dh of the tiles as two bf16 terms each, [tile][ranks, whole tiles][32 rows]
    const float *kept_h;
    uint16_t *left_h[2], *left_dh[2];
};

// A float as a sum of two bf16 values (16 bits of mantissa).  Where it is no number or too large the first says so alone.  One value would add an
// error as large as the results' own rounding; the second costs a matrix instruction, which kernels that wait for memory have to spare.
__device__ __forceinline__ void split(float v, uint16_t *hi, uint16_t *lo)
{
    *hi = mw_f32_to_bf16(v);
    const float rest = v - mw_bf16_to_f32(*hi);
    *lo = rest - rest == 0.0f ? mw_f32_to_bf16(rest) : 0;
}

constexpr int kWaves = 4, kBlock = kWaves * 64;

// This workgroup's tile: its adapter (-1: there is no such tile) and its rows; part: place of the first one's h, where they lie in order.
struct tile_rows { int32_t adapter, count, part; int32_t row[32]; };
__device__ __forceinline__ void find_tile(const adapt_args &p, int n_rows, tile_rows &t)
{
    const int tid = threadIdx.x, index = (int)blockIdx.x, step = (int)blockDim.x;
    if (p.tiles) {
        const adapt_tile a = p.tiles[index];
        if (tid < a.count) t.row[tid] = p.order[a.first + tid];
        if (tid == 0) { t.adapter = a.adapter; t.count = a.count; t.part = a.first; }
        mw_lds_barrier();
        return;
    }
    // Few rows, one a thread: bins counted, the bin that the index-th tile is of, and of its rows those of the tile, in order.
    __shared__ uint32_t hist[kBins], scratch[17];
    __shared__ uint32_t bin_of_tile, first_of_tile, in_wave[16];
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = p.n;
    int b = -1;
    if (tid < p.T) {
        const int id = p.ids[tid];
        b = id < 0 || id >= n ? n : id;
        if (p.flags && (id < -1 || id >= n) && index == 0 && blockIdx.y == 0) atomicOr(p.flags, MW_FLAG_BAD_ADAPTER);
    }
    for (int i = tid; i <= n; i += step) hist[i] = 0;
    if (tid == 0) { t.adapter = -1; t.count = 0; t.part = -1; }
    mw_lds_barrier();
    if (b >= 0) atomicAdd(&hist[b], 1u);
    mw_lds_barrier();
    uint32_t before = 0;
    for (int i0 = 0; i0 <= n; i0 += step) {
        const uint32_t c = i0 + tid <= n ? hist[i0 + tid] : 0u, k = (c + (uint32_t)n_rows - 1) / (uint32_t)n_rows;
        uint32_t all;
        const uint32_t at = before + mw_block_exscan(k, scratch, &all);
        if ((uint32_t)index >= at && (uint32_t)index < at + k) {
            const uint32_t first = ((uint32_t)index - at) * (uint32_t)n_rows;
            bin_of_tile = (uint32_t)(i0 + tid);
            first_of_tile = first;
            t.adapter = i0 + tid;
            t.count = (int)min(c - first, (uint32_t)n_rows);
        }
        before += all;
    }
    mw_lds_barrier();
    if (t.adapter < 0) return;
    const bool mine = b == (int)bin_of_tile;
    const unsigned long long those = __ballot(mine);
    if (lane == 0) in_wave[wave] = (uint32_t)__popcll(those);
    mw_lds_barrier();
    int rank = __popcll(those & ((1ull << lane) - 1)) - (int)first_of_tile;
    for (int w = 0; w < wave; ++w) rank += (int)in_wave[w];
    if (mine && rank >= 0 && rank < t.count) t.row[rank] = tid;
    mw_lds_barrier();
}

// Place of a row's h in the parts: rows of tiles that were found in the ids are where they are.
__device__ __forceinline__ int64_t part_of(const tile_rows &t, int col) { return t.part >= 0 ? t.part + col : t.row[col]; }

// h: kM tiles of 16 ranks by kCols tiles of 16 rows.  grid: (tile, slice of n_in).  Few tiles are cut into slices of four waves; where the
// tiles alone fill the card as many waves share a tile's columns out as their pieces of LDS leave room for, and there is one
// slice, or nearly.  us of mw_adapt, four waves / many: 300 rows of 4 adapters, rank 16, 17.4 / 19.6; 700 of 8 19.8 / 22.3; 1500 of 8, rank 32,
// 32.2 / 32.1; 2443 of 8, rank 64, 7168 to 7168, 75.9 / 62.3.
template <int kM> constexpr int kManyWaves = kM <= 2 ? 16 : kM == 4 ? 8 : 4;
template <int kM, int kCols, int kWaves>
__global__ __launch_bounds__(kWaves * 64) void k_adapt_down(adapt_args p)
{
    constexpr int kBlock = kWaves * 64;
    constexpr int kRanks = kM * 16, kRows = kCols * 16, kDepth = kM == 1 || (kWaves == 4 && kM == 2) ? 3 : 2;
    constexpr int kPartBytes = kWaves * kRows * kRanks * 4, kStageBytes = kWaves * kWaveLds<kM>;
    __shared__ __align__(16) char lds[kPartBytes > kStageBytes ? kPartBytes : kStageBytes];
    __shared__ tile_rows t;
    find_tile(p, kRows, t);
    const int adapter = __builtin_amdgcn_readfirstlane(t.adapter);
    if (adapter < 0 || adapter == p.n) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), n = lane & 15, g = lane >> 4, l8 = lane >> 3;
    const int start = (int)blockIdx.y * p.slice;
    const uint32_t piece = (uint32_t)(lane & 7) * 16 + (uint32_t)start * 2;
    operands<false, kM, kCols, 2, 1> o;
    o.w = array_at(p.a + (int64_t)adapter * p.rank * p.n_in);
    o.b[0] = array_at(p.x);
    o.limit = min(p.slice, p.n_in - start);
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = c * 16 + i * 8 + l8;
            o.col[c][0][i] = (uint32_t)((int64_t)t.row[at < t.count ? at : 0] * p.x_stride * 2) + piece;
        }
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) o.row[m][i] = (uint32_t)(min(m * 16 + i * 8 + l8, p.rank - 1) * p.n_in * 2) + piece;
    f32x4 acc[kM][kCols] = {};
    stream<false, kM, kCols, 2, 1, kWaves, kDepth, kOnceCols>(o, wave, lane, lds + wave * kWaveLds<kM>, acc);
    float *part = (float *)lds;             // [wave][row][rank]
    __syncthreads();
#pragma unroll
    for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int c = 0; c < kCols; ++c) *(f32x4 *)&part[((wave * kRows) + c * 16 + n) * kRanks + m * 16 + g * 4] = acc[m][c];
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * kRanks / 4; i += kBlock) {
        if (i / (kRanks / 4) >= t.count) break;
        f32x4 v = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += *(const f32x4 *)&part[w * kRows * kRanks + i * 4];
        *(f32x4 *)&p.part[((int64_t)blockIdx.y * p.T + part_of(t, i / (kRanks / 4))) * kRanks + i % (kRanks / 4) * 4] = v;
    }
}

// Eight ranks of a row of h as operands: the sum of the slices' parts, or what a forward pass kept, times the adapter's factor.
__device__ __forceinline__ void operand_of(const float (&v)[8], float scale, bf16x8 *hi, bf16x8 *lo)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        uint16_t a, b;
        split(v[e] * scale, &a, &b);
        (*hi)[e] = __builtin_bit_cast(__bf16, a);
        (*lo)[e] = __builtin_bit_cast(__bf16, b);
    }
}

// y: a wave takes 64 columns of the output at a time, as four tiles of rows of B; h is the other side, in registers.  What comes out goes
// through LDS so that base and y are read and written in whole cache lines.  grid: (tile, slice of n_out)
template <int kM, int kCols>
__global__ __launch_bounds__(kBlock) void k_adapt_up(adapt_args p)
{
    constexpr int kRanks = kM * 16, kRows = kCols * 16, kSteps = (kRanks + 31) / 32;
    constexpr int kLoads = 2 * kM;                          // 16-byte pieces a lane has of 64 rows of B, at most
    constexpr int kOutPitch = 68;                           // floats from row to row of the result in LDS
    constexpr int kWorkBytes = 64 * (kRanks * 2 + 16) > kRows * kOutPitch * 4 ? 64 * (kRanks * 2 + 16) : kRows * kOutPitch * 4;
    __shared__ __align__(16) char work[kWaves][kWorkBytes];
    __shared__ tile_rows t;
    find_tile(p, kRows, t);
    const int adapter = __builtin_amdgcn_readfirstlane(t.adapter), count = __builtin_amdgcn_readfirstlane(t.count);
    if (adapter < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4, l8 = lane >> 3, q8 = (lane & 7) * 8;
    const int c_from = (int)blockIdx.y * p.out_slice, c_to = min(c_from + p.out_slice, p.n_out);
    if (adapter == p.n) {                                   // rows without an adapter
        // A wave two rows, four pieces of each a lane on the way at a time.
        for (int r = wave * 2; r < count; r += kWaves * 2) {
            const int64_t row[2] = {__builtin_amdgcn_readfirstlane(t.row[r]), __builtin_amdgcn_readfirstlane(t.row[min(r + 1, count - 1)])};
            for (int c0 = c_from + lane * 8; c0 < c_to; c0 += 4 * 512) {
                u32x4 v[2][4] = {};
                if (p.base) {
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[i][j] = mw_ld16((const u32x4 *)(p.base + row[i] * p.base_stride + min(c0 + j * 512, c_to - 8)));
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (c0 + j * 512 < c_to && r + i < count) *(u32x4 *)(p.out + row[i] * p.out_stride + c0 + j * 512) = v[i][j];
            }
        }
        if (p.h && blockIdx.y == 0)
            for (int i = tid; i < count * p.rank; i += kBlock) p.h[(int64_t)t.row[i / p.rank] * p.rank + i % p.rank] = 0.0f;
        return;
    }
    const array b = array_at(p.b + (int64_t)adapter * p.rank * p.n_out), base = array_at(p.base ? p.base : p.out), out = array_at(p.out);
    char *mine = work[wave];
    const int pitch = p.rank * 2 + 16, n_loads = p.rank / 8;
    const uint32_t b_end = (uint32_t)p.n_out * (uint32_t)p.rank;
    uint32_t base_at[2 * kCols], out_at[2 * kCols];         // a lane's rows
#pragma unroll
    for (int i = 0; i < 2 * kCols; ++i) {
        const bool live = i * 8 + l8 < count;
        const int64_t row = t.row[live ? i * 8 + l8 : 0];
        base_at[i] = p.base ? (uint32_t)(row * p.base_stride * 2) : kNowhere;
        out_at[i] = live ? (uint32_t)(row * p.out_stride * 2) : kNowhere;
    }
    u32x4 bw[2][kLoads], was[2][2 * kCols];
    auto load = [&](int c, u32x4 (&bq)[kLoads], u32x4 (&wq)[2 * kCols]) {
        const uint32_t at = c < c_to ? 0u : kNowhere;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {                  // (past the last row of B: nothing)
            const uint32_t e = (uint32_t)((i * 64 + lane) * 8);
            bq[i] = load16<false>(b, at | (i < n_loads && (uint32_t)(c * p.rank) + e < b_end ? (uint32_t)(c * p.rank) * 2 + e * 2 : kNowhere));
        }
#pragma unroll
        for (int i = 0; i < 2 * kCols; ++i) wq[i] = load16<true>(base, at | (c + q8 < c_to ? base_at[i] + (uint32_t)(c + q8) * 2 : kNowhere));
    };
    load(c_from + wave * 64, bw[0], was[0]);               // (on their way while h is added up)
    // h of the lane's rows: eight ranks a step.  Past the last rank or row: zeros, from past the parts' end.
    const float scale = p.scale ? p.scale[adapter] : 1.0f;
    const array parts = array_at(p.part);
    bf16x8 hv[kCols][kSteps], lv[kCols][kSteps];
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
        const int col = i * 16 + n;
        const int64_t at = part_of(t, col < count ? col : 0);
        float v[kSteps][8] = {};
#pragma unroll 4
        for (int s = 0; s < p.n_slices; ++s)
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int r = k * 32 + g * 8;
                const uint32_t from = col < count && r < p.rank ? (uint32_t)((((int64_t)s * p.T + at) * kRanks + r) * 4) : kNowhere;
                const f32x4 v0 = __builtin_bit_cast(f32x4, load16<false>(parts, from)), v1 = __builtin_bit_cast(f32x4, load16<false>(parts, from + 16));
#pragma unroll
                for (int e = 0; e < 4; ++e) { v[k][e] += v0[e]; v[k][4 + e] += v1[e]; }
            }
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int r = k * 32 + g * 8;
            operand_of(v[k], scale, &hv[i][k], &lv[i][k]);
            if (p.h && blockIdx.y == 0 && wave == 0 && col < count && r < p.rank) {
#pragma unroll
                for (int e = 0; e < 8; ++e) p.h[(int64_t)t.row[col] * p.rank + r + e] = v[k][e];
            }
        }
    }
    if constexpr (kCols == 2) {
        // What k_adapt_grads needs of the tile: h and dh as [rank][32 rows], by the first and the last slice's workgroup.
        uint16_t *left = (uint16_t *)work;                  // [term][row][rank]
        constexpr int kStep = kRanks + 8;                   // (rows start on different banks)
        for (int side = 0; side < 2; ++side) {
            if (!p.kept_h || (int)blockIdx.y != (side == 0 ? 0 : (int)gridDim.y - 1)) continue;
            if (wave == 0) {
#pragma unroll
                for (int i = 0; i < kCols; ++i)
#pragma unroll
                    for (int k = 0; k < kSteps; ++k) {
                        const int r = k * 32 + g * 8, col = i * 16 + n;
                        bf16x8 hi = hv[i][k], lo = lv[i][k];
                        if (side == 1) {
                            float v[8] = {};
                            if (col < count && r < p.rank) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[e] = p.kept_h[(int64_t)t.row[col] * p.rank + r + e];
                            }
                            operand_of(v, scale, &hi, &lo);
                        }
                        if (r < kRanks) {
                            *(bf16x8 *)&left[col * kStep + r] = hi;
                            *(bf16x8 *)&left[(kRows + col) * kStep + r] = lo;
                        }
                    }
            }
            mw_lds_barrier();
            for (int i = tid; i < kRanks * 4 * 2; i += kBlock) {
                const uint16_t *from = left + (i & 1) * kRows * kStep;
                const int r = i >> 3, q = (i >> 1 & 3) * 8;
                uint32_t v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = from[(q + 2 * j) * kStep + r] | (uint32_t)from[(q + 2 * j + 1) * kStep + r] << 16;
                *(u32x4 *)((side == 0 ? p.left_dh : p.left_h)[i & 1] + ((int64_t)blockIdx.x * kRanks + r) * 32 + q) = u32x4{v[0], v[1], v[2], v[3]};
            }
            mw_lds_barrier();
        }
    }
    uint32_t to_lds[kLoads];                                // where a lane's pieces of B go in LDS
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int e = (i * 64 + lane) * 8;
        to_lds[i] = (uint32_t)(e / p.rank * pitch + e % p.rank * 2);
    }
    const bf16x8 none = {};
    for (int c0 = c_from + wave * 64; c0 < c_to; c0 += 2 * kWaves * 64) {
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            const int c = c0 + d * kWaves * 64;
            load(c + kWaves * 64, bw[d ^ 1], was[d ^ 1]);
            wave_order();
#pragma unroll
            for (int i = 0; i < kLoads; ++i) if (i < n_loads) *(u32x4 *)(mine + to_lds[i]) = bw[d][i];
            wave_order();
            f32x4 acc[4][kCols] = {};
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int kk = k * 32 + g * 8;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const bf16x8 bv = kk < p.rank ? *(const bf16x8 *)(mine + (q * 16 + n) * pitch + kk * 2) : none;
#pragma unroll
                    for (int i = 0; i < kCols; ++i) {
                        acc[q][i] = mma(bv, lv[i][k], acc[q][i]);
                        acc[q][i] = mma(bv, hv[i][k], acc[q][i]);
                    }
                }
            }
            float *res = (float *)mine;                     // [row][64 columns]
            wave_order();
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < kCols; ++i) *(f32x4 *)&res[(i * 16 + n) * kOutPitch + q * 16 + g * 4] = acc[q][i];
            wave_order();
#pragma unroll
            for (int i = 0; i < 2 * kCols; ++i) {
                const f32x4 v0 = *(const f32x4 *)&res[(i * 8 + l8) * kOutPitch + q8], v1 = *(const f32x4 *)&res[(i * 8 + l8) * kOutPitch + q8 + 4];
                const bf16x8 w = __builtin_bit_cast(bf16x8, was[d][i]);
                bf16x8 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) { y[e] = (__bf16)((float)w[e] + v0[e]); y[4 + e] = (__bf16)((float)w[4 + e] + v1[e]); }
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, y), out, c + q8 < c_to && out_at[i] != kNowhere ? out_at[i] + (uint32_t)(c + q8) * 2 : kNowhere, 0, 2);
            }
        }
    }
}

// Eight vectors of eight 16-bit values, transposed.
__device__ __forceinline__ void transpose8(u32x4 (&v)[8])
{
    bf16x8 in[8], r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) in[i] = __builtin_bit_cast(bf16x8, v[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) r[i][j] = in[j][i];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(u32x4, r[i]);
}

struct grad_args {
    const int32_t *order, *tile_at; const adapt_tile *tiles;
    int32_t rank, ranks;                   // ranks: whole tiles of 16
    // side 0: d_a[m][c] = sum_t (c dh)[t][m] x[t][c];  side 1: d_b[c][m] = sum_t (c h)[t][m] dy[t][c]
    const uint16_t *left[2][2];            // [side][term]: [tile][ranks][32 rows]
    const uint16_t *right[2]; int64_t stride[2]; int32_t width[2];
    uint16_t *out[2];
};

// grid: (128 columns, adapter, side and piece of 32 ranks).  The waves take an adapter's tiles of 32 rows in turn: a tile is one
// matrix instruction deep.  Rows of x are loaded as they lie, 256 bytes of four rows an instruction, and turned in registers: a lane has eight
// rows of eight columns, and the columns' vectors over the rows are operands.  The instance of 32 ranks has 264 registers, 96 of them sums: one
// workgroup a CU, with nothing beside it while it waits for its loads.  That bounds it, and rows that are one workgroup's alone.
constexpr int kGradWaves = 4;
template <int kM>
__global__ __launch_bounds__(kGradWaves * 64) void k_adapt_grads(grad_args p)
{
    __shared__ __align__(16) float part[kGradWaves * 8 * 256];
    constexpr int kTurned = kM * 16 + 8;                        // [128 columns][ranks]
    __shared__ __align__(16) uint16_t turned[128 * kTurned];
    const int side = blockIdx.z & 1, r0 = (blockIdx.z >> 1) * 32, ad = blockIdx.y, c0 = blockIdx.x * 128, width = p.width[side];
    if (c0 >= width) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), n = lane & 15, g = lane >> 4;
    const int tile0 = p.tile_at[ad], tile1 = p.tile_at[ad + 1];
    const int64_t stride = p.stride[side];
    const int col = c0 + n * 8;
    if (tile0 == tile1) {                                       // an adapter without rows: zeros
        const u32x4 zero = {};
        for (int i = threadIdx.x; i < 128 * kM * 2; i += kGradWaves * 64) {
            if (side == 0) {
                const int r = r0 + i / 16, c = c0 + i % 16 * 8;
                if (r < p.rank && c < width) *(u32x4 *)(p.out[0] + ((int64_t)ad * p.rank + r) * width + c) = zero;
            } else {
                const int c = c0 + i / (kM * 2), r = r0 + i % (kM * 2) * 8;
                if (c < width && r < p.rank) *(u32x4 *)(p.out[1] + ((int64_t)ad * width + c) * p.rank + r) = zero;
            }
        }
        return;
    }
    const array right = array_at(p.right[side]), hi_of = array_at(p.left[side][0]), lo_of = array_at(p.left[side][1]);
    const uint32_t c_at = col < width ? (uint32_t)col * 2 : kNowhere;
    f32x4 acc[kM][8] = {};
    u32x4 v[2][8], hi[2][kM], lo[2][kM];
    {
        const int first = p.tiles[tile0].first, end = p.tiles[tile1 - 1].first + p.tiles[tile1 - 1].count;     // the adapter's rows in the order
        int row[2][8];
        // A tile's rows, a step ahead of what is loaded of them; past the last tile nothing.
        auto rows = [&](int k, int (&rq)[8]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) rq[j] = p.order[min(first + (k - tile0) * 32 + g * 8 + j, end - 1)];
        };
        auto load = [&](int k, const int (&rq)[8], u32x4 (&vq)[8], u32x4 (&hq)[kM], u32x4 (&lq)[kM]) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                vq[j] = load16<false>(right, first + (k - tile0) * 32 + g * 8 + j < end && c_at != kNowhere ? (uint32_t)((int64_t)rq[j] * stride * 2) + c_at : kNowhere);
#pragma unroll
            for (int m = 0; m < kM; ++m) {
                const uint32_t at = k < tile1 ? (uint32_t)((k * p.ranks + r0 + m * 16 + n) * 64 + g * 16) : kNowhere;
                hq[m] = load16<false>(hi_of, at);
                lq[m] = load16<false>(lo_of, at);
            }
        };
        rows(tile0 + wave, row[0]);
        rows(tile0 + wave + kGradWaves, row[1]);
        load(tile0 + wave, row[0], v[0], hi[0], lo[0]);
        for (int k0 = tile0 + wave; k0 < tile1; k0 += 2 * kGradWaves) {
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                load(k0 + (d + 1) * kGradWaves, row[d ^ 1], v[d ^ 1], hi[d ^ 1], lo[d ^ 1]);
                rows(k0 + (d + 2) * kGradWaves, row[d]);
                transpose8(v[d]);
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        acc[m][j] = mma(__builtin_bit_cast(bf16x8, lo[d][m]), __builtin_bit_cast(bf16x8, v[d][j]), acc[m][j]);
                        acc[m][j] = mma(__builtin_bit_cast(bf16x8, hi[d][m]), __builtin_bit_cast(bf16x8, v[d][j]), acc[m][j]);
                    }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < kM; ++m) {
#pragma unroll
        for (int j = 0; j < 8; ++j) *(f32x4 *)&part[((wave * 8 + j) * 64 + lane) * 4] = acc[m][j];
        __syncthreads();
        if (wave == m % kGradWaves && col < width) {
            f32x4 s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[j] = *(const f32x4 *)&part[(j * 64 + lane) * 4];
#pragma unroll
                for (int w = 1; w < kGradWaves; ++w) s[j] += *(const f32x4 *)&part[((w * 8 + j) * 64 + lane) * 4];
            }
            const int r = r0 + m * 16 + g * 4;                  // (rank is a multiple of 8: four ranks are in or out together)
            if (r < p.rank) {
                if (side == 0) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        bf16x8 o;
#pragma unroll
                        for (int j = 0; j < 8; ++j) o[j] = (__bf16)s[j][i];
                        *(bf16x8 *)(p.out[0] + ((int64_t)ad * p.rank + r + i) * width + col) = o;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        bf16x4 o;
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[i] = (__bf16)s[j][i];
                        *(bf16x4 *)&turned[(n * 8 + j) * kTurned + m * 16 + g * 4] = o;
                    }
                }
            }
        }
        __syncthreads();
    }
    if (side == 1) {                                            // a column's ranks lie together: 16-byte pieces of them
        constexpr int kPieces = kM * 2;
        for (int i = threadIdx.x; i < 128 * kPieces; i += kGradWaves * 64) {
            const int at = i / kPieces, r = i % kPieces * 8;
            if (c0 + at < width && r0 + r < p.rank) *(u32x4 *)(p.out[1] + ((int64_t)ad * width + c0 + at) * p.rank + r0 + r) = *(const u32x4 *)&turned[at * kTurned + r];
        }
    }
}

int ranks_of(int32_t rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : rank <= 64 ? 64 : 128; }
constexpr int kMostSlices = 8;
constexpr int64_t kMostCus = 512;          // (rows times slices stay below rows + 128 times the CUs: a tile has at most 32 rows)

// Rows of a tile: 32 where adapters have 96 rows on average, and where the gradients want tiles one matrix instruction deep; else 16.  us of
// mw_adapt, 24 adapters of rank 16, 4096 to 4096, 16 / 32: 300 rows 19.0 / 22.1, 1200 22.9 / 26.2, 2400 29.8 / 30.0; of rank 64, 7168 to 4096: 1200 37.6 /
// 38.0, 2400 57.1 / 48.6; 40 of rank 128, 4000 rows 155 / 85.  8 of rank 32, 4096 to 7168, 800 rows 25.0 / 28.1: on the wrong side.
int tile_rows_of(const mw_adapters *s, int64_t rows, bool backward) { return backward || rows >= 96LL * s->n_adapters ? 32 : 16; }
int64_t most_tiles(const mw_adapters *s, int64_t rows, int tile_rows) { return rows / tile_rows + (s->n_adapters + 1LL < rows ? s->n_adapters + 1LL : rows); }

struct adapt_ws { int64_t order, tile_at, tiles, part, left[4], at, bt, total; };
adapt_ws adapt_layout(const mw_adapters *s, int64_t rows, bool backward)
{
    adapt_ws w;
    int64_t o = 0;
    const int64_t tiles = most_tiles(s, rows, 16), ranks = ranks_of(s->rank);
    w.order = o;   o += mw_align_up(4 * rows, 256);
    w.tile_at = o; o += mw_align_up(4 * (s->n_adapters + 2LL), 256);
    w.tiles = o;   o += mw_align_up((int64_t)sizeof(adapt_tile) * tiles, 256);
    w.part = o;    o += mw_align_up(4 * ranks * (rows * kMostSlices < rows + 128 * kMostCus ? rows * kMostSlices : rows + 128 * kMostCus), 256);
    for (int i = 0; i < 4; ++i) { w.left[i] = o; o += backward ? mw_align_up(2 * most_tiles(s, rows, 32) * ranks * 32, 256) : 0; }
    w.at = o;      o += backward ? mw_align_up(2LL * s->n_adapters * s->rank * s->n_in, 256) : 0;
    w.bt = o;      o += backward ? mw_align_up(2LL * s->n_adapters * s->rank * s->n_out, 256) : 0;
    w.total = o;
    return w;
}

int32_t adapters_ready(const mw_adapters *s)
{
    if (!s || s->n_adapters < 1 || s->rank < 1 || s->n_in < 1 || s->n_out < 1) return MW_ERR_INVALID_ARG;
    if (s->n_adapters > MW_ADAPT_MAX_ADAPTERS || s->rank > MW_ADAPT_MAX_RANK) return MW_ERR_UNSUPPORTED;
    if (s->rank % 8 != 0 || s->n_in % 8 != 0 || s->n_out % 8 != 0 || s->n_in > (1 << 20) || s->n_out > (1 << 20)) return MW_ERR_UNSUPPORTED;
    return MW_OK;
}
// a bf16 matrix of rows in one piece each
bool rows_ready(const void *p, int64_t stride, int32_t width) { return p && ((uintptr_t)p & 15u) == 0 && stride >= width && stride % 8 == 0; }
// Places in such a matrix are 32-bit, below 2^31 bytes.  (Divided: a product of any stride with the rows may pass 64 bits.)
bool too_far(int64_t stride, int32_t rows) { return rows > 0 && stride > (1LL << 30) / rows; }

order_args order_of(const mw_adapters *s, const int32_t *ids, int32_t T, char *ws, const adapt_ws &w, int tile_rows, uint32_t *flags)
{
    order_args o;
    o.ids = ids; o.T = T; o.n = s->n_adapters; o.tile_rows = tile_rows; o.most_tiles = (int32_t)most_tiles(s, T, tile_rows);
    o.order = (int32_t *)(ws + w.order); o.tile_at = (int32_t *)(ws + w.tile_at); o.tiles = (adapt_tile *)(ws + w.tiles);
    o.flags = flags;
    return o;
}
// Slices of a tile's `width` columns, so that all workgroups are resident at once.
int64_t slices(int64_t width, int64_t workgroups, int64_t tiles, int64_t least, int64_t most)
{
    int64_t n = workgroups / tiles;
    const int64_t all = (width + least - 1) / least;
    n = n < all ? n : all;
    n = n < most ? n : most;
    return n < 1 ? 1 : n;
}
// Workgroups of k_adapt_up that a CU holds at once, by their registers and LDS.
template <int kM, int kCols>
int resident_up()
{
    static const int n = [] {
        int most = 0;
        return hipOccupancyMaxActiveBlocksPerMultiprocessor(&most, k_adapt_up<kM, kCols>, kBlock, 0) == hipSuccess && most > 0 ? most : 1;
    }();
    return n;
}
template <int kM, int kCols>
void launch_both(adapt_args p, bool few, int64_t tiles, int n_cu, hipStream_t st)
{
    // A sixteenth more than a CU holds: `tiles` counts the most there can be, and a few that come later cost less than a slice fewer of all.  us with / without
    // it, and by LDS alone: 8192 rows of 8 adapters, rank 32, 7168 to 4096, 66.2 / 70.4 / 66.0; 5000 of 16, rank 64, 2880 to 5120, 59.9 / 65.0 / 67.2; 2000 of 4, rank
    // 128, 4096 to 4096, 42.6 / 46.2 / 57.9; 2443 of 8, rank 64, 7168 to 7168, 54.2 / 54.1 / 61.7.
    const int64_t m = slices(p.n_out, (int64_t)resident_up<kM, kCols>() * n_cu * 17 / 16, tiles, 256, 4096);
    p.out_slice = (int32_t)mw_align_up((p.n_out + m - 1) / m, 64);
    const dim3 down((uint32_t)tiles, (uint32_t)p.n_slices), up((uint32_t)tiles, (uint32_t)((p.n_out + p.out_slice - 1) / p.out_slice));
    if (few) hipLaunchKernelGGL((k_adapt_down<kM, kCols, 4>), down, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_adapt_down<kM, kCols, kManyWaves<kM>>), down, dim3(kManyWaves<kM> * 64), 0, st, p);
    hipLaunchKernelGGL((k_adapt_up<kM, kCols>), up, dim3(kBlock), 0, st, p);
}
// h and y.  p.a to p.out, p.T, p.h, and p.tiles or p.ids are set.
int32_t launch_adapt(adapt_args p, const mw_adapters *s, int tile_rows, char *ws, const adapt_ws &w, int n_cu, hipStream_t st)
{
    p.scale = s->scale_dev; p.n = s->n_adapters; p.rank = s->rank;
    p.part = (float *)(ws + w.part);
    const int64_t tiles = most_tiles(s, p.T, tile_rows);
    const bool few = tiles * 8 <= n_cu, wide = tile_rows == 32;
    const int64_t n = few ? slices(p.n_in, 3LL * n_cu, tiles, 1024, kMostSlices) : slices(p.n_in, n_cu, tiles, 2048, kMostSlices);      // (a wave has two spans at least)
    p.slice = (int32_t)mw_align_up((p.n_in + n - 1) / n, 64);
    p.n_slices = (p.n_in + p.slice - 1) / p.slice;
    switch (ranks_of(p.rank)) {
    case 16: if (wide) launch_both<1, 2>(p, few, tiles, n_cu, st); else launch_both<1, 1>(p, few, tiles, n_cu, st); break;
    case 32: if (wide) launch_both<2, 2>(p, few, tiles, n_cu, st); else launch_both<2, 1>(p, few, tiles, n_cu, st); break;
    case 64: if (wide) launch_both<4, 2>(p, few, tiles, n_cu, st); else launch_both<4, 1>(p, few, tiles, n_cu, st); break;
    default: if (wide) launch_both<8, 2>(p, few, tiles, n_cu, st); else launch_both<8, 1>(p, few, tiles, n_cu, st); break;
    }
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
int32_t cus_of_current_device(int *n)
{
    int dev = -1;
    MW_HIP_CHECK(hipGetDevice(&dev));
    MW_HIP_CHECK(hipDeviceGetAttribute(n, hipDeviceAttributeMultiprocessorCount, dev));
    if (*n < 1) *n = 256;
    if (*n > kMostCus) *n = kMostCus;
    return MW_OK;
}

}  // namespace

extern "C" MW_API int32_t mw_adapt_workspace_bytes(const mw_adapters *adapters, int32_t max_rows, int32_t backward, int64_t *out_bytes)
{
    if (!out_bytes || max_rows < 0) return MW_ERR_INVALID_ARG;
    const int32_t rc = adapters_ready(adapters);
    if (rc != MW_OK) return rc;
    if (max_rows > MW_ADAPT_MAX_ROWS) return MW_ERR_CAPACITY;
    *out_bytes = adapt_layout(adapters, max_rows, backward != 0).total;
    return MW_OK;
}

extern "C" MW_API int32_t mw_adapt(const mw_adapters *adapters, const void *x_dev, int64_t x_stride, const int32_t *adapter_ids_dev,
                                   int32_t n_rows, const void *base_dev, int64_t base_stride, void *out_dev, int64_t out_stride,
                                   float *h_dev, uint32_t *error_flags_dev, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    const int32_t rc = adapters_ready(adapters);
    if (rc != MW_OK) return rc;
    const mw_adapters &s = *adapters;
    if (n_rows < 0) return MW_ERR_INVALID_ARG;
    if (n_rows > MW_ADAPT_MAX_ROWS) return MW_ERR_CAPACITY;
    if (n_rows == 0) return MW_OK;
    if (!s.a_dev || !s.b_dev || (((uintptr_t)s.a_dev | (uintptr_t)s.b_dev) & 15u) || ((uintptr_t)s.scale_dev & 3u)) return MW_ERR_INVALID_ARG;
    if (!adapter_ids_dev || !rows_ready(x_dev, x_stride, s.n_in) || !rows_ready(out_dev, out_stride, s.n_out)) return MW_ERR_INVALID_ARG;
    if (base_dev && !rows_ready(base_dev, base_stride, s.n_out)) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)h_dev | (uintptr_t)error_flags_dev | (uintptr_t)adapter_ids_dev) & 3u) return MW_ERR_INVALID_ARG;
    const adapt_ws w = adapt_layout(adapters, n_rows, false);
    if (!workspace_dev || ((uintptr_t)workspace_dev & 255u) || workspace_bytes < w.total) return MW_ERR_WORKSPACE;
    if (too_far(x_stride, n_rows) || too_far(out_stride, n_rows) || (base_dev && too_far(base_stride, n_rows))) return MW_ERR_UNSUPPORTED;
    int n_cu = 0;
    const int32_t rd = cus_of_current_device(&n_cu);
    if (rd != MW_OK) return rd;
    const hipStream_t st = (hipStream_t)stream;
    char *ws = (char *)workspace_dev;
    adapt_args p = {};
    p.a = (const uint16_t *)s.a_dev; p.b = (const uint16_t *)s.b_dev; p.T = n_rows; p.n_in = s.n_in; p.n_out = s.n_out;
    p.x = (const uint16_t *)x_dev; p.x_stride = x_stride;
    p.base = (const uint16_t *)base_dev; p.base_stride = base_stride;
    p.out = (uint16_t *)out_dev; p.out_stride = out_stride;
    p.h = h_dev;
    const int tile = tile_rows_of(adapters, n_rows, false);
    // Up to 256 rows every workgroup finds its tile in the ids: a launch less.  us, so / with the order first: 1 row 10.9 / 14.3, 256 of 64 adapters 17.0 /
    // 20.3 (rank 16, 4096 to 4096); 64 of 24, rank 16, 7168 to 7168, 14.2 / 17.9; 64 of 24, rank 64, 16.9 / 20.5; 256 of 4, rank 32, 7168 to 4096, 17.0 /
    // 20.2; 200 of 16, rank 128, 24.4 / 27.9.
    if (n_rows <= kBlock) {
        p.ids = adapter_ids_dev;
        p.flags = error_flags_dev;
    } else {
        const order_args o = order_of(adapters, adapter_ids_dev, n_rows, ws, w, tile, error_flags_dev);
        hipLaunchKernelGGL(k_adapt_order, dim3(1), dim3(kOrderBlock), order_lds_bytes(o.n), st, o);
        MW_HIP_CHECK(hipGetLastError());
        p.order = o.order; p.tiles = o.tiles;
    }
    return launch_adapt(p, adapters, tile, ws, w, n_cu, st);
}

extern "C" MW_API int32_t mw_adapt_backward(const mw_adapters *adapters, const void *x_dev, int64_t x_stride, const int32_t *adapter_ids_dev,
                                            int32_t n_rows, const float *h_dev, const void *dy_dev, int64_t dy_stride,
                                            const void *dx_base_dev, int64_t dx_base_stride, void *dx_dev, int64_t dx_stride,
                                            void *da_dev, void *db_dev, uint32_t *error_flags_dev, void *workspace_dev,
                                            int64_t workspace_bytes, void *stream)
{
    const int32_t rc = adapters_ready(adapters);
    if (rc != MW_OK) return rc;
    const mw_adapters &s = *adapters;
    if (n_rows < 0) return MW_ERR_INVALID_ARG;
    if (n_rows > MW_ADAPT_MAX_ROWS) return MW_ERR_CAPACITY;
    if (!s.a_dev || !s.b_dev || (((uintptr_t)s.a_dev | (uintptr_t)s.b_dev) & 15u) || ((uintptr_t)s.scale_dev & 3u)) return MW_ERR_INVALID_ARG;
    if (!da_dev || !db_dev || (((uintptr_t)da_dev | (uintptr_t)db_dev) & 15u)) return MW_ERR_INVALID_ARG;
    if (n_rows > 0) {
        if (!adapter_ids_dev || !h_dev || !rows_ready(x_dev, x_stride, s.n_in) || !rows_ready(dy_dev, dy_stride, s.n_out)) return MW_ERR_INVALID_ARG;
        if (!rows_ready(dx_dev, dx_stride, s.n_in)) return MW_ERR_INVALID_ARG;
        if (dx_base_dev && !rows_ready(dx_base_dev, dx_base_stride, s.n_in)) return MW_ERR_INVALID_ARG;
        if (((uintptr_t)h_dev | (uintptr_t)error_flags_dev | (uintptr_t)adapter_ids_dev) & 3u) return MW_ERR_INVALID_ARG;
    }
    const adapt_ws w = adapt_layout(adapters, n_rows, true);
    if (!workspace_dev || ((uintptr_t)workspace_dev & 255u) || workspace_bytes < w.total) return MW_ERR_WORKSPACE;
    if (too_far(x_stride, n_rows) || too_far(dy_stride, n_rows) || too_far(dx_stride, n_rows) || (dx_base_dev && too_far(dx_base_stride, n_rows))) return MW_ERR_UNSUPPORTED;
    int n_cu = 0;
    const int32_t rd = cus_of_current_device(&n_cu);
    if (rd != MW_OK) return rd;
    char *ws = (char *)workspace_dev;
    const hipStream_t st = (hipStream_t)stream;
    const order_args o = order_of(adapters, adapter_ids_dev, n_rows, ws, w, 32, error_flags_dev);
    const transpose_args ta = {(const uint16_t *)s.a_dev, (uint16_t *)(ws + w.at), s.rank, s.n_in};
    const transpose_args tb = {(const uint16_t *)s.b_dev, (uint16_t *)(ws + w.bt), s.n_out, s.rank};
    const int64_t pieces = s.n_adapters * (pieces_of(ta) + pieces_of(tb)), blocks = pieces < kMostPieces ? pieces : kMostPieces;
    hipLaunchKernelGGL(k_adapt_prepare, dim3(n_rows > 0 ? (uint32_t)(1 + blocks) : 1u), dim3(kOrderBlock), order_lds_bytes(o.n), st, o, ta, tb);
    MW_HIP_CHECK(hipGetLastError());
    uint16_t *left[4];
    for (int i = 0; i < 4; ++i) left[i] = (uint16_t *)(ws + w.left[i]);
    if (n_rows > 0) {
        adapt_args p = {};
        p.a = tb.out; p.b = ta.out; p.T = n_rows; p.n_in = s.n_out; p.n_out = s.n_in;
        p.x = (const uint16_t *)dy_dev; p.x_stride = dy_stride;
        p.base = (const uint16_t *)dx_base_dev; p.base_stride = dx_base_stride;
        p.out = (uint16_t *)dx_dev; p.out_stride = dx_stride;
        p.kept_h = h_dev;
        p.order = o.order; p.tiles = o.tiles;
        for (int i = 0; i < 2; ++i) { p.left_dh[i] = left[i]; p.left_h[i] = left[2 + i]; }
        const int32_t ra = launch_adapt(p, adapters, 32, ws, w, n_cu, st);
        if (ra != MW_OK) return ra;
    }
    grad_args q;
    q.order = o.order; q.tile_at = o.tile_at; q.tiles = o.tiles; q.rank = s.rank; q.ranks = ranks_of(s.rank);
    for (int i = 0; i < 2; ++i) { q.left[0][i] = left[i]; q.left[1][i] = left[2 + i]; }
    q.right[0] = (const uint16_t *)x_dev; q.stride[0] = x_stride; q.width[0] = s.n_in; q.out[0] = (uint16_t *)da_dev;
    q.right[1] = (const uint16_t *)dy_dev; q.stride[1] = dy_stride; q.width[1] = s.n_out; q.out[1] = (uint16_t *)db_dev;
    const int32_t widest = s.n_in > s.n_out ? s.n_in : s.n_out;
    const dim3 grid((uint32_t)((widest + 127) / 128), (uint32_t)s.n_adapters, (uint32_t)(2 * ((q.ranks + 31) / 32)));
    if (q.ranks == 16) hipLaunchKernelGGL((k_adapt_grads<1>), grid, dim3(kGradWaves * 64), 0, st, q);
    else hipLaunchKernelGGL((k_adapt_grads<2>), grid, dim3(kGradWaves * 64), 0, st, q);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
