// mw_adapt, mw_adapt_backward: low-rank adapters of many requests beside a shared projection.
//
//   y_t  = base_t + c_a B_a h_t,   h_t = A_a x_t                       a: the adapter of row t
//   dh_t = B_a^T dy_t,   dx_t = dx_base_t + c_a A_a^T dh_t,   dA_a = c_a sum_t dh_t x_t^T,   dB_a = c_a sum_t dy_t h_t^T
//
// Rows are put in order of their adapters first (stable, so sums over an adapter's rows have one order).  A workgroup then takes up to
// 32 rows of one adapter through both products: x once, h in LDS only, base and y once.  The gradient of the input is the same
// walk with the transposed factors.
#include "mw_math.h"

namespace {

constexpr int kTileRows = 32;
constexpr int kOrderBlock = 512, kOrderWaves = kOrderBlock / 64;
constexpr int kBins = MW_ADAPT_MAX_ADAPTERS + 1;       // the last: rows without an adapter

struct adapt_tile { int32_t adapter, first, count, reserved0; };      // adapter == n_adapters: rows without one

// One workgroup.  order: rows by (adapter, row); start[b]: first of adapter b's in it; tiles of at most kTileRows.
__global__ __launch_bounds__(kOrderBlock) void k_adapt_order(const int32_t *__restrict__ ids, int T, int n, int32_t *__restrict__ order,
                                                             int32_t *__restrict__ start, adapt_tile *__restrict__ tiles,
                                                             int32_t *__restrict__ n_tiles, uint32_t *__restrict__ flags)
{
    __shared__ uint32_t hist[kOrderWaves][kBins];
    __shared__ uint32_t row_at[kBins + 1], tile_at[kBins + 1];
    __shared__ uint32_t scratch[17];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = tid; i < kOrderWaves * (n + 1); i += kOrderBlock) hist[i / (n + 1)][i % (n + 1)] = 0;
    __syncthreads();
    const int per = ((T + kOrderWaves - 1) / kOrderWaves + 63) / 64 * 64;      // a wave's rows, in pieces of 64
    const int lo = wave * per, hi = min(T, lo + per);
    bool wrong = false;
    for (int at = lo; at < hi; at += 64) {
        const int t = at + lane;
        if (t < hi) {
            const int id = ids[t];
            wrong |= id < -1 || id >= n;
            atomicAdd(&hist[wave][id < 0 || id >= n ? n : id], 1u);
        }
    }
    if (flags && wrong) atomicOr(flags, MW_FLAG_BAD_ADAPTER);
    __syncthreads();
    // places: bins in order, in a bin the waves in order
    constexpr int kPer = (kBins + kOrderBlock - 1) / kOrderBlock;
    uint32_t rows[kPer], rsum = 0, tsum = 0, total;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = tid * kPer + i;
        rows[i] = 0;
        if (b <= n)
            for (int w = 0; w < kOrderWaves; ++w) rows[i] += hist[w][b];
        rsum += rows[i];
        tsum += (rows[i] + kTileRows - 1) / kTileRows;
    }
    uint32_t r = mw_block_exscan(rsum, scratch, &total);
    uint32_t k = mw_block_exscan(tsum, scratch, &total);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int b = tid * kPer + i;
        if (b <= n) {
            row_at[b] = r;
            tile_at[b] = k;
            start[b] = (int32_t)r;
            uint32_t p = r;
            for (int w = 0; w < kOrderWaves; ++w) {
                const uint32_t c = hist[w][b];
                hist[w][b] = p;
                p += c;
            }
        }
        r += rows[i];
        k += (rows[i] + kTileRows - 1) / kTileRows;
    }
    if (tid == 0) {
        row_at[n + 1] = (uint32_t)T;
        tile_at[n + 1] = total;
        start[n + 1] = T;
        *n_tiles = (int32_t)total;
    }
    __syncthreads();
    for (int i = tid; i < (int)total; i += kOrderBlock) {      // the bin a tile is of: the last that starts at or before it
        int at = 0, end = n + 1;
        while (end - at > 1) {
            const int mid = (at + end) / 2;
            if (tile_at[mid] <= (uint32_t)i) at = mid; else end = mid;
        }
        const int first = (int)row_at[at] + (i - (int)tile_at[at]) * kTileRows;
        tiles[i] = adapt_tile{at, first, min(kTileRows, (int)row_at[at + 1] - first), 0};
    }
    int bits = 0;
    while ((1 << bits) <= n) ++bits;
    for (int at = lo; at < hi; at += 64) {
        const int t = at + lane;
        const bool live = t < hi;
        int b = n;
        if (live) {
            b = ids[t];
            if (b < 0 || b >= n) b = n;
        }
        unsigned long long same = __ballot(live);              // the piece's rows of the same adapter
        for (int i = 0; i < bits; ++i) {
            const unsigned long long set = __ballot((b >> i) & 1);
            same &= (b >> i) & 1 ? set : ~set;
        }
        if (live) {
            const int before = __popcll(same & ((1ull << lane) - 1));
            const uint32_t p = hist[wave][b] + (uint32_t)before;
            order[p] = t;
            __builtin_amdgcn_wave_barrier();
            if (before == 0) hist[wave][b] += (uint32_t)__popcll(same);
        }
    }
}

struct adapt_args {
    const int32_t *order; const adapt_tile *tiles; const int32_t *n_tiles; const int32_t *start;
    const uint16_t *a, *b;                 // [n][rank][n_in], [n][n_out][rank]
    const float *scale;                    // [n]
    int32_t n, rank, n_in, n_out;
    const uint16_t *x; int64_t x_stride;
    const uint16_t *base; int64_t base_stride;     // or null
    uint16_t *out; int64_t out_stride;
    float *h;                              // [T][rank] or null
};

__device__ __forceinline__ bf16x8 load8(const uint16_t *p, bool live)
{
    const bf16x8 zero = {};
    return live ? *(const bf16x8 *)p : zero;
}
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// A float as a sum of two bf16 values (16 bits of mantissa).  Where it is no number or too large the first says so alone.
__device__ __forceinline__ void split(float v, uint16_t *hi, uint16_t *lo)
{
    *hi = mw_f32_to_bf16(v);
    const float rest = v - mw_bf16_to_f32(*hi);
    *lo = rest - rest == 0.0f ? mw_f32_to_bf16(rest) : 0;
}

constexpr int kWaves = 8, kBlock = kWaves * 64;
constexpr int kPartTiles = 2;              // tiles of 16 ranks whose partial sums are in LDS at a time
template <int kM>                          // tiles of 16 ranks
__global__ __launch_bounds__(kBlock) void k_adapt(adapt_args p)
{
    constexpr int kRanks = kM * 16, kStep = kRanks + 8;         // (rows of h in LDS start on different banks)
    constexpr int kParts = kM < kPartTiles ? kM : kPartTiles;
    __shared__ __align__(16) float part[kWaves * kParts * 16 * kTileRows];
    __shared__ __align__(16) uint16_t h_hi[kTileRows * kStep], h_lo[kTileRows * kStep];
    if ((int)blockIdx.x >= *p.n_tiles) return;
    const adapt_tile t = p.tiles[blockIdx.x];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    if (t.adapter == p.n) {                                     // rows without an adapter
        const int pieces = p.n_out / 8;
        for (int i = tid; i < t.count * pieces; i += kBlock) {
            const int64_t row = p.order[t.first + i / pieces];
            const int c = i % pieces * 8;
            *(bf16x8 *)(p.out + row * p.out_stride + c) = load8(p.base + row * p.base_stride + c, p.base != nullptr);
        }
        if (p.h)
            for (int i = tid; i < t.count * p.rank; i += kBlock) p.h[(int64_t)p.order[t.first + i / p.rank] * p.rank + i % p.rank] = 0.0f;
        return;
    }
    const uint16_t *a = p.a + (int64_t)t.adapter * p.rank * p.n_in, *b = p.b + (int64_t)t.adapter * p.rank * p.n_out;
    int64_t row[2];
    bool live[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        live[i] = i * 16 + n < t.count;
        row[i] = p.order[t.first + (live[i] ? i * 16 + n : 0)];
    }
    {   // h: the waves share the columns out in chunks of 128
        f32x4 acc[kM][2] = {};
        for (int c = wave * 128; c < p.n_in; c += kWaves * 128) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = c + j * 32 + g * 8;
                bf16x8 xv[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) xv[i] = load8(p.x + row[i] * p.x_stride + k, live[i] && k < p.n_in);
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                    const bf16x8 av = load8(a + (int64_t)min(m * 16 + n, p.rank - 1) * p.n_in + k, k < p.n_in);
#pragma unroll
                    for (int i = 0; i < 2; ++i) acc[m][i] = mma(av, xv[i], acc[m][i]);
                }
            }
        }
        const float scale = p.scale ? p.scale[t.adapter] : 1.0f;
#pragma unroll
        for (int m0 = 0; m0 < kM; m0 += kParts) {
            // part [wave][tile][row][16 ranks]
#pragma unroll
            for (int m = 0; m < kParts; ++m)
#pragma unroll
                for (int i = 0; i < 2; ++i) *(f32x4 *)&part[((wave * kParts + m) * kTileRows + i * 16 + n) * 16 + g * 4] = acc[m0 + m][i];
            __syncthreads();
            for (int o = tid; o < kParts * kTileRows * 16; o += kBlock) {
                float v = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) v += part[w * kParts * kTileRows * 16 + o];
                const int r = (m0 + o / (kTileRows * 16)) * 16 + o % 16, col = o / 16 % kTileRows;
                const bool real = r < p.rank && col < t.count;
                if (p.h && real) p.h[(int64_t)p.order[t.first + col] * p.rank + r] = v;
                split(real ? v * scale : 0.0f, &h_hi[col * kStep + r], &h_lo[col * kStep + r]);
            }
            __syncthreads();
        }
    }
    // y: a wave takes 64 columns of the output at a time.  Row m of tile q is column (m / 4) * 16 + q * 4 + m % 4, so that a lane ends
    // up with 16 neighbouring columns of its row.
    for (int c = wave * 64; c < p.n_out; c += kWaves * 64) {
        f32x4 acc[4][2] = {};
        const int col = c + (n >> 2) * 16 + (n & 3);
#pragma unroll
        for (int k = 0; k < kRanks; k += 32) {
            bf16x8 hv[2], lv[2], bv[4];
            const int kk = k + g * 8;
#pragma unroll
            for (int q = 0; q < 4; ++q) bv[q] = load8(b + (int64_t)(col + q * 4) * p.rank + kk, col + q * 4 < p.n_out && kk < p.rank);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                hv[i] = load8(&h_hi[(i * 16 + n) * kStep + kk], kk < kRanks);
                lv[i] = load8(&h_lo[(i * 16 + n) * kStep + kk], kk < kRanks);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    acc[q][i] = mma(bv[q], lv[i], acc[q][i]);
                    acc[q][i] = mma(bv[q], hv[i], acc[q][i]);
                }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int at = c + g * 16 + half * 8;
                if (!live[i] || at >= p.n_out) continue;
                const bf16x8 was = load8(p.base + row[i] * p.base_stride + at, p.base != nullptr);
                bf16x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (__bf16)((float)was[e] + acc[half * 2 + e / 4][i][e % 4]);
                *(bf16x8 *)(p.out + row[i] * p.out_stride + at) = v;
            }
    }
}

// [n][rows][cols] -> [n][cols][rows] of 16-bit values.  grid: (64 columns, 64 rows, matrix).
__global__ __launch_bounds__(256) void k_adapt_transpose(const uint16_t *__restrict__ in, uint16_t *__restrict__ out, int rows, int cols)
{
    __shared__ uint16_t tile[64][66];
    const int64_t at = (int64_t)blockIdx.z * rows * cols;
    const int c0 = blockIdx.x * 64, r0 = blockIdx.y * 64;
    for (int i = threadIdx.x; i < 4096; i += 256) {
        const int r = i >> 6, c = i & 63;
        if (r0 + r < rows && c0 + c < cols) tile[r][c] = in[at + (int64_t)(r0 + r) * cols + c0 + c];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 4096; i += 256) {
        const int c = i >> 6, r = i & 63;
        if (r0 + r < rows && c0 + c < cols) out[at + (int64_t)(c0 + c) * rows + r0 + r] = tile[r][c];
    }
}

// Eight vectors of eight 16-bit values, transposed.
__device__ __forceinline__ void transpose8(bf16x8 (&v)[8])
{
    bf16x8 r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) r[i][j] = v[j][i];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = r[i];
}

struct grad_args {
    const int32_t *order, *start;
    const float *scale;
    int32_t rank;
    // z 0: d_a[m][c] = c sum_t dh[t][m] x[t][c];  z 1: d_b[c][m] = c sum_t h[t][m] dy[t][c]
    const float *left[2];                  // [T][rank]
    const uint16_t *right[2]; int64_t stride[2]; int32_t width[2];
    uint16_t *out[2];
};

// grid: (128 columns, adapter, {dA, dB} x pieces of 64 ranks).  The waves take 32 of the adapter's rows at a time.
constexpr int kGradWaves = 4;
template <int kM>
__global__ __launch_bounds__(kGradWaves * 64) void k_adapt_grads(grad_args p)
{
    __shared__ __align__(16) float part[kGradWaves * 8 * 256];
    const int side = blockIdx.z & 1, r0 = (blockIdx.z >> 1) * 64, ad = blockIdx.y, c0 = blockIdx.x * 128, width = p.width[side];
    if (c0 >= width) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const int first = p.start[ad], count = p.start[ad + 1] - first;
    const float *left = p.left[side];
    const uint16_t *right = p.right[side];
    const int64_t stride = p.stride[side];
    const int col = c0 + n * 8;
    f32x4 acc[kM][8] = {};
    for (int k = wave * 32; k < count; k += kGradWaves * 32) {
        bf16x8 v[8];
        bf16x8 hi[kM], lo[kM];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool live = k + g * 8 + j < count;
            const int64_t row = p.order[first + (live ? k + g * 8 + j : 0)];
            v[j] = load8(right + row * stride + col, live && col < width);
#pragma unroll
            for (int m = 0; m < kM; ++m) {
                const int r = r0 + m * 16 + n;
                uint16_t a, b;
                split(live && r < p.rank ? left[row * p.rank + r] : 0.0f, &a, &b);
                hi[m][j] = __builtin_bit_cast(__bf16, a);
                lo[m][j] = __builtin_bit_cast(__bf16, b);
            }
        }
        transpose8(v);
#pragma unroll
        for (int m = 0; m < kM; ++m)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                acc[m][j] = mma(lo[m], v[j], acc[m][j]);
                acc[m][j] = mma(hi[m], v[j], acc[m][j]);
            }
    }
    const float scale = p.scale ? p.scale[ad] : 1.0f;
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
                        for (int j = 0; j < 8; ++j) o[j] = (__bf16)(scale * s[j][i]);
                        *(bf16x8 *)(p.out[0] + ((int64_t)ad * p.rank + r + i) * width + col) = o;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        bf16x4 o;
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[i] = (__bf16)(scale * s[j][i]);
                        *(bf16x4 *)(p.out[1] + ((int64_t)ad * width + col + j) * p.rank + r) = o;
                    }
                }
            }
        }
        __syncthreads();
    }
}

struct adapt_ws { int64_t order, start, tiles, n_tiles, dh, at, bt, total; };
adapt_ws adapt_layout(const mw_adapters *s, int64_t rows, bool backward)
{
    adapt_ws w;
    int64_t o = 0;
    w.order = o;   o += mw_align_up(4 * rows, 256);
    w.start = o;   o += mw_align_up(4 * (s->n_adapters + 2LL), 256);
    w.tiles = o;   o += mw_align_up((int64_t)sizeof(adapt_tile) * (rows / kTileRows + s->n_adapters + 1), 256);
    w.n_tiles = o; o += 256;
    w.dh = o;      o += backward ? mw_align_up(4 * rows * s->rank, 256) : 0;
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

void launch_order(const mw_adapters *s, const int32_t *ids, int32_t T, char *ws, const adapt_ws &w, uint32_t *flags, adapt_args *p, hipStream_t st)
{
    hipLaunchKernelGGL(k_adapt_order, dim3(1), dim3(kOrderBlock), 0, st, ids, T, s->n_adapters, (int32_t *)(ws + w.order), (int32_t *)(ws + w.start),
                       (adapt_tile *)(ws + w.tiles), (int32_t *)(ws + w.n_tiles), flags);
    p->order = (const int32_t *)(ws + w.order); p->start = (const int32_t *)(ws + w.start);
    p->tiles = (const adapt_tile *)(ws + w.tiles); p->n_tiles = (const int32_t *)(ws + w.n_tiles);
    p->scale = s->scale_dev; p->n = s->n_adapters; p->rank = s->rank;
}
void launch_adapt(const adapt_args &p, int32_t T, hipStream_t st)
{
    const dim3 grid((uint32_t)(T / kTileRows + (p.n + 1 < T ? p.n + 1 : T)));       // tiles there can be at most
    if (p.rank <= 16) hipLaunchKernelGGL((k_adapt<1>), grid, dim3(kBlock), 0, st, p);
    else if (p.rank <= 32) hipLaunchKernelGGL((k_adapt<2>), grid, dim3(kBlock), 0, st, p);
    else if (p.rank <= 64) hipLaunchKernelGGL((k_adapt<4>), grid, dim3(kBlock), 0, st, p);
    else hipLaunchKernelGGL((k_adapt<8>), grid, dim3(kBlock), 0, st, p);
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
    const hipStream_t st = (hipStream_t)stream;
    adapt_args p;
    launch_order(adapters, adapter_ids_dev, n_rows, (char *)workspace_dev, w, error_flags_dev, &p, st);
    MW_HIP_CHECK(hipGetLastError());
    p.a = (const uint16_t *)s.a_dev; p.b = (const uint16_t *)s.b_dev; p.n_in = s.n_in; p.n_out = s.n_out;
    p.x = (const uint16_t *)x_dev; p.x_stride = x_stride;
    p.base = (const uint16_t *)base_dev; p.base_stride = base_stride;
    p.out = (uint16_t *)out_dev; p.out_stride = out_stride;
    p.h = h_dev;
    launch_adapt(p, n_rows, st);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
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
    char *ws = (char *)workspace_dev;
    const hipStream_t st = (hipStream_t)stream;
    adapt_args p;
    launch_order(adapters, adapter_ids_dev, n_rows, ws, w, error_flags_dev, &p, st);
    MW_HIP_CHECK(hipGetLastError());
    uint16_t *at = (uint16_t *)(ws + w.at), *bt = (uint16_t *)(ws + w.bt);
    float *dh = (float *)(ws + w.dh);
    if (n_rows > 0) {
        const uint32_t r64 = (uint32_t)((s.rank + 63) / 64), n = (uint32_t)s.n_adapters;
        hipLaunchKernelGGL(k_adapt_transpose, dim3((uint32_t)((s.n_in + 63) / 64), r64, n), dim3(256), 0, st, (const uint16_t *)s.a_dev, at, s.rank, s.n_in);
        hipLaunchKernelGGL(k_adapt_transpose, dim3(r64, (uint32_t)((s.n_out + 63) / 64), n), dim3(256), 0, st, (const uint16_t *)s.b_dev, bt, s.n_out, s.rank);
        MW_HIP_CHECK(hipGetLastError());
        p.a = bt; p.b = at; p.n_in = s.n_out; p.n_out = s.n_in;
        p.x = (const uint16_t *)dy_dev; p.x_stride = dy_stride;
        p.base = (const uint16_t *)dx_base_dev; p.base_stride = dx_base_stride;
        p.out = (uint16_t *)dx_dev; p.out_stride = dx_stride;
        p.h = dh;
        launch_adapt(p, n_rows, st);
        MW_HIP_CHECK(hipGetLastError());
    }
    grad_args q;
    q.order = p.order; q.start = p.start; q.scale = s.scale_dev; q.rank = s.rank;
    q.left[0] = dh; q.right[0] = (const uint16_t *)x_dev; q.stride[0] = x_stride; q.width[0] = s.n_in; q.out[0] = (uint16_t *)da_dev;
    q.left[1] = h_dev; q.right[1] = (const uint16_t *)dy_dev; q.stride[1] = dy_stride; q.width[1] = s.n_out; q.out[1] = (uint16_t *)db_dev;
    const int32_t widest = s.n_in > s.n_out ? s.n_in : s.n_out;
    const dim3 grid((uint32_t)((widest + 127) / 128), (uint32_t)s.n_adapters, (uint32_t)(2 * ((s.rank + 63) / 64)));
    if (s.rank <= 16) hipLaunchKernelGGL((k_adapt_grads<1>), grid, dim3(kGradWaves * 64), 0, st, q);
    else if (s.rank <= 32) hipLaunchKernelGGL((k_adapt_grads<2>), grid, dim3(kGradWaves * 64), 0, st, q);
    else hipLaunchKernelGGL((k_adapt_grads<4>), grid, dim3(kGradWaves * 64), 0, st, q);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
