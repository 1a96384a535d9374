// mw_ffn, mw_ffn_backward: the experts of the rows that a dispatch brought.
#include "mw_tile.h"
#include "mw_ffn.h"

namespace {

// ---- h = silu(x Wg^T) * (x Wu^T) --------------------------------------------------------------------------------
struct up_args {
    row_groups g;
    const uint16_t *x; int64_t x_stride;
    const uint16_t *w;                      // [n][2][I][H]
    uint16_t *h, *kept;                     // [rows][I], [rows][2][I] or null
    int32_t H, I, p_tiles;
};
// Half of a tile's columns are gate rows, half the up rows beside them: a lane then holds both values of an element.
template <int kP, int kQ>
__global__ __launch_bounds__(kTileThreads, kP * kQ > 128 * 128 ? 1 : 2) void k_ffn_up(up_args a)
{
    typedef tile_product<kP, kQ, false, false, false> product;
    __shared__ __attribute__((aligned(1024))) char lds[product::kLds];
    tile_at at;
    if (!find_tile<kQ>(a.g, a.p_tiles, at)) return;
    const int col0 = at.p * (kP / 2);
    tile_feed<kP, false, false> fp;
    tile_feed<kQ, false, false> fq;
    fp.rows((const char *)(a.w + ((int64_t)at.e * 2 * a.I + col0) * a.H), a.H, [&](int r) {
        const int in = r % (kP / 2), up = in / (kP / 4), col = r / (kP / 2) * (kP / 4) + tile_column(in % (kP / 4));
        return col0 + col < a.I ? (uint32_t)(up * a.I + col) * (uint32_t)a.H * 2 : kNowhereAt;
    });
    fq.rows((const char *)(a.x + at.first * a.x_stride), a.H, [&](int r) { return r < at.rows ? (uint32_t)r * (uint32_t)a.x_stride * 2 : kNowhereAt; });
    product t;
    t.run(fp, fq, (a.H + 63) / 64, (lds_char *)lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < product::kNQ; ++j) {
        const int row = (wave >> 1) * (kQ / 2) + j * 32 + (lane & 31);
        if (row >= at.rows) continue;
        uint16_t *h = a.h + (at.first + row) * a.I, *kept = a.kept ? a.kept + (at.first + row) * 2 * a.I : nullptr;
#pragma unroll
        for (int i = 0; i < product::kNP / 2; ++i)
#pragma unroll
            for (int s = 0; s < 16; s += 8) {
                const int col = col0 + (wave & 1) * (kP / 4) + i * 32 + (lane >> 5) * 16 + s;
                if (col >= a.I) continue;
                float gate[8], up[8], v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    gate[e] = t.acc[i][j][s + e];
                    up[e] = t.acc[i + product::kNP / 2][j][s + e];
                    v[e] = gate[e] * tile_sigmoid(gate[e]) * up[e];
                }
                store_bf16<8>(h + col, v);
                if (kept) {
                    store_bf16<8>(kept + col, gate);
                    store_bf16<8>(kept + a.I + col, up);
                }
            }
    }
}

// ---- rows times a matrix: y = w h Wd^T, dx = [dg du] [Wg; Wu] ---------------------------------------------------
struct rows_args {
    row_groups g;
    const uint16_t *x; int64_t x_stride;    // [rows][K]
    const uint16_t *w;                      // [n][N][K], kTr: [n][K][N]
    const float *row_weights;               // or null
    uint16_t *y; int64_t y_stride;
    int32_t K, N, p_tiles;
};
template <int kP>
__device__ __forceinline__ void columns_from(tile_feed<kP, true, false> &fp, const uint16_t *w, int col0, int K, int N)
{
    fp.lines((const char *)(w + col0), K, (int64_t)N * 2, N - col0);
}
template <int kP>
__device__ __forceinline__ void columns_from(tile_feed<kP, false, false> &fp, const uint16_t *w, int col0, int K, int N)
{
    fp.rows((const char *)(w + (int64_t)col0 * K), K, [&](int r) {
        const int col = tile_column(r);
        return col0 + col < N ? (uint32_t)col * (uint32_t)K * 2 : kNowhereAt;
    });
}
template <int kP, int kQ, bool kTr>
__global__ __launch_bounds__(kTileThreads, kP * kQ > 128 * 128 ? 1 : 2) void k_ffn_rows(rows_args a)
{
    typedef tile_product<kP, kQ, kTr, false, false> product;
    __shared__ __attribute__((aligned(1024))) char lds[product::kLds];
    tile_at at;
    if (!find_tile<kQ>(a.g, a.p_tiles, at)) return;
    const int col0 = at.p * kP;
    const uint16_t *w = a.w + (int64_t)at.e * a.N * a.K;
    tile_feed<kP, kTr, false> fp;
    tile_feed<kQ, false, false> fq;
    columns_from(fp, w, col0, a.K, a.N);
    fq.rows((const char *)(a.x + at.first * a.x_stride), a.K, [&](int r) { return r < at.rows ? (uint32_t)r * (uint32_t)a.x_stride * 2 : kNowhereAt; });
    product t;
    t.run(fp, fq, (a.K + 63) / 64, (lds_char *)lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < product::kNQ; ++j) {
        const int row = (wave >> 1) * (kQ / 2) + j * 32 + (lane & 31);
        if (row >= at.rows) continue;
        const float weight = a.row_weights ? a.row_weights[at.first + row] : 1.0f;
        uint16_t *y = a.y + (at.first + row) * a.y_stride;
#pragma unroll
        for (int i = 0; i < product::kNP; ++i) {
            constexpr int kPiece = kTr ? 4 : 8;
#pragma unroll
            for (int s = 0; s < 16; s += kPiece) {
                const int col = col0 + (wave & 1) * (kP / 2) + i * 32 + (kTr ? s * 2 + (lane >> 5) * 4 : (lane >> 5) * 16 + s);
                if (col >= a.N) continue;
                float v[kPiece];
#pragma unroll
                for (int e = 0; e < kPiece; ++e) v[e] = a.row_weights ? weight * t.acc[i][j][s + e] : t.acc[i][j][s + e];
                store_bf16<kPiece>(y + col, v);
            }
        }
    }
}

// ---- da = dy Wd, and what follows from it element by element ------------------------------------------------------
struct act_args {
    row_groups g;
    const uint16_t *dy; int64_t dy_stride;
    const uint16_t *down;                   // [n][H][I]
    const float *row_weights;               // or null
    const uint16_t *kept;                   // [rows][2][I]
    uint16_t *act, *d_gate_up;              // [rows][I], [rows][2][I]
    float *parts;                           // [parts][part_rows] or null: sums of da h over a wave's columns
    int64_t part_rows;
    int32_t H, I, p_tiles;
};
template <int kP, int kQ>
__global__ __launch_bounds__(kTileThreads, kP * kQ > 128 * 128 ? 1 : 2) void k_ffn_act(act_args a)
{
    typedef tile_product<kP, kQ, true, false, false> product;
    __shared__ __attribute__((aligned(1024))) char lds[product::kLds];
    tile_at at;
    if (!find_tile<kQ>(a.g, a.p_tiles, at)) return;
    const int col0 = at.p * kP;
    tile_feed<kP, true, false> fp;
    tile_feed<kQ, false, false> fq;
    fp.lines((const char *)(a.down + (int64_t)at.e * a.H * a.I + col0), a.H, (int64_t)a.I * 2, a.I - col0);
    fq.rows((const char *)(a.dy + at.first * a.dy_stride), a.H, [&](int r) { return r < at.rows ? (uint32_t)r * (uint32_t)a.dy_stride * 2 : kNowhereAt; });
    product t;
    t.run(fp, fq, (a.H + 63) / 64, (lds_char *)lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < product::kNQ; ++j) {
        const int row = (wave >> 1) * (kQ / 2) + j * 32 + (lane & 31);
        float sum = 0.0f;
        if (row < at.rows) {
            const float weight = a.row_weights ? a.row_weights[at.first + row] : 1.0f;
            const uint16_t *kept = a.kept + (at.first + row) * 2 * a.I;
            uint16_t *act = a.act + (at.first + row) * a.I, *d = a.d_gate_up + (at.first + row) * 2 * a.I;
#pragma unroll
            for (int i = 0; i < product::kNP; ++i)
#pragma unroll
                for (int s = 0; s < 16; s += 4) {
                    const int col = col0 + (wave & 1) * (kP / 2) + i * 32 + s * 2 + (lane >> 5) * 4;
                    if (col >= a.I) continue;
                    const bf16x4 gate = *(const bf16x4 *)(kept + col), up = *(const bf16x4 *)(kept + a.I + col);
                    float h[4], dg[4], du[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float g = (float)gate[e], u = (float)up[e], sig = tile_sigmoid(g), silu = g * sig, da = t.acc[i][j][s + e], dh = weight * da;
                        sum += da * silu * u;
                        h[e] = weight * silu * u;
                        dg[e] = dh * u * (sig + silu * (1.0f - sig));
                        du[e] = dh * silu;
                    }
                    store_bf16<4>(act + col, h);
                    store_bf16<4>(d + col, dg);
                    store_bf16<4>(d + a.I + col, du);
                }
        }
        if (a.parts) {
            sum += __shfl_xor(sum, 32);
            if (row < at.rows && lane < 32) a.parts[(int64_t)(at.p * 2 + (wave & 1)) * a.part_rows + at.first + row] = sum;
        }
    }
}
// d_row_weights: a row's sums, in the order of their columns.
__global__ __launch_bounds__(256) void k_ffn_weights(row_groups g, const float *parts, int n_parts, float *out)
{
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x, end = min(max(g.offsets[g.n], (int64_t)0), g.n_rows);
    if (row >= end) return;
    float v = 0.0f;
    for (int i = 0; i < n_parts; ++i) v += parts[(int64_t)i * g.n_rows + row];
    out[row] = v;
}

// ---- gradients of matrices: out[q][p] = sum over a run's rows of q's value times p's ---------------------------------
struct grads_args {
    row_groups g;
    const uint16_t *q, *p; int64_t q_stride, p_stride;
    uint16_t *out;                          // [n][M][N]
    int32_t M, N, p_tiles, q_tiles;
};
template <int kP, int kQ>
__global__ __launch_bounds__(kTileThreads, kP * kQ > 128 * 128 ? 1 : 2) void k_ffn_grads(grads_args a)
{
    typedef tile_product<kP, kQ, true, true, false> product;
    __shared__ __attribute__((aligned(1024))) char lds[product::kLds];
    const uint32_t each = (uint32_t)a.p_tiles * (uint32_t)a.q_tiles;
    uint32_t tile, pt, qt;
    if (!tile_of_workgroup(each * (uint32_t)a.g.n, tile)) return;
    const int e = (int)(tile / each);
    tile_in_block(tile - (uint32_t)e * each, a.p_tiles, a.q_tiles, pt, qt);
    const int q0 = (int)qt * kQ, p0 = (int)pt * kP;
    int64_t first, end;
    group_bounds(a.g, e, first, end);
    const int rows = (int)(end - first);
    tile_feed<kP, true, false> fp;
    tile_feed<kQ, true, false> fq;
    fp.lines((const char *)(a.p + first * a.p_stride + p0), rows, a.p_stride * 2, a.N - p0);
    fq.lines((const char *)(a.q + first * a.q_stride + q0), rows, a.q_stride * 2, a.M - q0);
    product t;
    t.run(fp, fq, (rows + 63) / 64, (lds_char *)lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint16_t *out = a.out + (int64_t)e * a.M * a.N;
#pragma unroll
    for (int j = 0; j < product::kNQ; ++j) {
        const int row = q0 + (wave >> 1) * (kQ / 2) + j * 32 + (lane & 31);
        if (row >= a.M) continue;
#pragma unroll
        for (int i = 0; i < product::kNP; ++i)
#pragma unroll
            for (int s = 0; s < 16; s += 4) {
                const int col = p0 + (wave & 1) * (kP / 2) + i * 32 + s * 2 + (lane >> 5) * 4;
                if (col >= a.N) continue;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = t.acc[i][j][s + e];
                store_bf16<4>(out + (int64_t)row * a.N + col, v);
            }
    }
}

// ---- entry points -----------------------------------------------------------------------------------------------------
int64_t pieces(int64_t n, int64_t each) { return (n + each - 1) / each; }

struct ffn_ws { int64_t act, d_gate_up, parts, codes, scales, total; };
ffn_ws ffn_layout(const mw_experts *e, int32_t hidden, int64_t rows, bool backward)
{
    ffn_ws w = {};
    int64_t o = 0;
    auto take = [&](int64_t bytes) { const int64_t at = o; o += mw_align_up(bytes, 256); return at; };
    w.act = take(2 * rows * e->inter);
    if (backward) {
        w.d_gate_up = take(4 * rows * e->inter);
        w.parts = take(4 * rows * pieces(e->inter, 64));
    }
    if (e->format == MW_WEIGHT_INT8_CHANNEL) {
        w.codes = take(rows * (hidden > e->inter ? hidden : e->inter));
        w.scales = take(4 * rows);
    }
    w.total = o > 0 ? o : 256;
    return w;
}

int32_t ffn_ready(const mw_ctx *ctx, const mw_experts *e, bool backward)
{
    if (!e || ctx->cfg.n_experts < 1 || e->inter < 1) return MW_ERR_INVALID_ARG;
    const bool int8 = e->format == MW_WEIGHT_INT8_CHANNEL;
    if (ctx->cfg.row_format == MW_ROW_BYTES || e->format == MW_ROW_FP8_E4M3_BLOCK128 || (int8 && backward)) return MW_ERR_UNSUPPORTED;
    if (!int8 && e->format != MW_ROW_BF16) return MW_ERR_INVALID_ARG;
    if (!int8 && (e->gate_up_scale_dev || e->down_scale_dev)) return MW_ERR_INVALID_ARG;
    const int32_t unit = int8 ? 16 : 8;          // rows of whole 16-byte pieces
    if (ctx->cfg.hidden % unit != 0 || e->inter % unit != 0 || e->inter > (1 << 20)) return MW_ERR_UNSUPPORTED;
    // places inside an expert's matrices are 32-bit, below 2^31
    if (2LL * (int8 ? 1 : 2) * ctx->cfg.hidden * e->inter > (2LL << 30)) return MW_ERR_UNSUPPORTED;
    if (int8 && (ctx->cfg.hidden > MW_INT8_MAX_IN || e->inter > MW_INT8_MAX_IN)) return MW_ERR_UNSUPPORTED;
    if (ctx->n_local > 0 && (!e->gate_up_dev || !e->down_dev || (int8 && (!e->gate_up_scale_dev || !e->down_scale_dev)))) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)e->gate_up_dev | (uintptr_t)e->down_dev) & 15u) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)e->gate_up_scale_dev | (uintptr_t)e->down_scale_dev) & 3u) return MW_ERR_INVALID_ARG;
    return MW_OK;
}
// A matrix of bf16 rows of the caller's.
bool rows_fit(const void *p, int64_t stride, int64_t width) { return p && !((uintptr_t)p & 15u) && stride >= width && stride % 8 == 0; }
template <int kP, int kQ>
int32_t launch_up(up_args a, hipStream_t s)
{
    a.p_tiles = (int32_t)pieces(a.I, kP / 2);
    const uint32_t grid = tile_grid(most_tiles(a.g.n_rows, a.g.n, kQ) * a.p_tiles);
    if (!grid) return MW_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((k_ffn_up<kP, kQ>), dim3(grid), dim3(kTileThreads), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
template <int kP, int kQ, bool kTr>
int32_t launch_rows(rows_args a, hipStream_t s)
{
    a.p_tiles = (int32_t)pieces(a.N, kP);
    const uint32_t grid = tile_grid(most_tiles(a.g.n_rows, a.g.n, kQ) * a.p_tiles);
    if (!grid) return MW_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((k_ffn_rows<kP, kQ, kTr>), dim3(grid), dim3(kTileThreads), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
template <int kP, int kQ>
int32_t launch_act(act_args a, hipStream_t s, int *n_parts)
{
    a.p_tiles = (int32_t)pieces(a.I, kP);
    const uint32_t grid = tile_grid(most_tiles(a.g.n_rows, a.g.n, kQ) * a.p_tiles);
    if (!grid) return MW_ERR_UNSUPPORTED;
    *n_parts = a.p_tiles * 2;
    hipLaunchKernelGGL((k_ffn_act<kP, kQ>), dim3(grid), dim3(kTileThreads), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
template <int kP, int kQ>
int32_t launch_grads(grads_args a, hipStream_t s)
{
    a.p_tiles = (int32_t)pieces(a.N, kP);
    a.q_tiles = (int32_t)pieces(a.M, kQ);
    const uint32_t grid = tile_grid((int64_t)a.p_tiles * a.q_tiles * a.g.n);
    if (!grid) return MW_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((k_ffn_grads<kP, kQ>), dim3(grid), dim3(kTileThreads), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}

}  // namespace

extern "C" MW_API int32_t mw_ffn_workspace_bytes(mw_ctx *ctx, const mw_experts *experts, int64_t max_rows, int32_t backward, int64_t *out_bytes)
{
    if (!ctx || !out_bytes || max_rows < 0) return MW_ERR_INVALID_ARG;
    const int32_t rc = ffn_ready(ctx, experts, backward != 0);
    if (rc != MW_OK) return rc;
    if (max_rows > MW_FFN_MAX_ROWS) return MW_ERR_CAPACITY;
    *out_bytes = ffn_layout(experts, ctx->cfg.hidden, max_rows, backward != 0).total;
    return MW_OK;
}

extern "C" MW_API int32_t mw_ffn(mw_ctx *ctx, const mw_experts *experts, const void *x_dev, int64_t x_stride, const int64_t *expert_offsets_dev,
                                 int64_t n_rows, const float *row_weights_dev, void *y_dev, int64_t y_stride, void *kept_dev,
                                 void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    if (!ctx || n_rows < 0) return MW_ERR_INVALID_ARG;
    int32_t rc = ffn_ready(ctx, experts, false);
    if (rc == MW_OK) rc = mw_on_device_of(ctx);
    if (rc != MW_OK) return rc;
    if (n_rows > MW_FFN_MAX_ROWS) return MW_ERR_CAPACITY;
    const bool int8 = experts->format == MW_WEIGHT_INT8_CHANNEL;
    const int32_t H = ctx->cfg.hidden, I = experts->inter;
    if (n_rows > 0 && (!rows_fit(x_dev, x_stride, H) || !rows_fit(y_dev, y_stride, H))) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)kept_dev & 15u) || ((uintptr_t)row_weights_dev & 3u) || ((uintptr_t)expert_offsets_dev & 7u) || !expert_offsets_dev) return MW_ERR_INVALID_ARG;
    if (int8 && kept_dev) return MW_ERR_INVALID_ARG;
    if (x_stride > MW_MAX_STRIDE || y_stride > MW_MAX_STRIDE) return MW_ERR_UNSUPPORTED;
    const ffn_ws w = ffn_layout(experts, H, n_rows, false);
    if (!workspace_dev || ((uintptr_t)workspace_dev & 255u) || workspace_bytes < w.total) return MW_ERR_WORKSPACE;
    if (n_rows == 0 || ctx->n_local == 0) return MW_OK;
    char *b = (char *)workspace_dev;
    const row_groups g = {expert_offsets_dev, n_rows, ctx->n_local};
    const hipStream_t s = (hipStream_t)stream;
    if (int8) return mw_ffn_int8(experts, H, x_dev, x_stride, expert_offsets_dev, ctx->n_local, n_rows, row_weights_dev, y_dev, y_stride, b + w.act, (int8_t *)(b + w.codes), (float *)(b + w.scales), s);
    up_args u = {g, (const uint16_t *)x_dev, x_stride, (const uint16_t *)experts->gate_up_dev, (uint16_t *)(b + w.act), (uint16_t *)kept_dev, H, I, 0};
    rows_args d = {g, (const uint16_t *)(b + w.act), I, (const uint16_t *)experts->down_dev, row_weights_dev, (uint16_t *)y_dev, y_stride, I, H, 0};
    const bool large = n_rows >= 192LL * g.n;
    rc = large ? launch_up<256, 256>(u, s) : launch_up<128, 64>(u, s);
    if (rc == MW_OK) rc = large ? launch_rows<256, 256, false>(d, s) : launch_rows<128, 64, false>(d, s);
    return rc;
}

extern "C" MW_API int32_t mw_ffn_backward(mw_ctx *ctx, const mw_experts *experts, const void *x_dev, int64_t x_stride, const int64_t *expert_offsets_dev,
                                          int64_t n_rows, const float *row_weights_dev, const void *kept_dev, const void *dy_dev, int64_t dy_stride,
                                          void *dx_dev, int64_t dx_stride, void *d_gate_up_dev, void *d_down_dev, float *d_row_weights_dev,
                                          void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    if (!ctx || n_rows < 0) return MW_ERR_INVALID_ARG;
    int32_t rc = ffn_ready(ctx, experts, true);
    if (rc == MW_OK) rc = mw_on_device_of(ctx);
    if (rc != MW_OK) return rc;
    if (n_rows > MW_FFN_MAX_ROWS) return MW_ERR_CAPACITY;
    const int32_t H = ctx->cfg.hidden, I = experts->inter;
    if (n_rows > 0 && (!rows_fit(x_dev, x_stride, H) || !rows_fit(dy_dev, dy_stride, H) || (dx_dev && !rows_fit(dx_dev, dx_stride, H)) || !kept_dev)) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)kept_dev | (uintptr_t)d_gate_up_dev | (uintptr_t)d_down_dev) & 15u) return MW_ERR_INVALID_ARG;
    if ((((uintptr_t)row_weights_dev | (uintptr_t)d_row_weights_dev) & 3u) || ((uintptr_t)expert_offsets_dev & 7u) || !expert_offsets_dev) return MW_ERR_INVALID_ARG;
    if (x_stride > MW_MAX_STRIDE || dy_stride > MW_MAX_STRIDE || (dx_dev && dx_stride > MW_MAX_STRIDE)) return MW_ERR_UNSUPPORTED;
    const ffn_ws w = ffn_layout(experts, H, n_rows, true);
    if (!workspace_dev || ((uintptr_t)workspace_dev & 255u) || workspace_bytes < w.total) return MW_ERR_WORKSPACE;
    if (ctx->n_local == 0) return MW_OK;
    char *b = (char *)workspace_dev;
    const row_groups g = {expert_offsets_dev, n_rows, ctx->n_local};
    const hipStream_t s = (hipStream_t)stream;
    uint16_t *act = (uint16_t *)(b + w.act), *d_act = (uint16_t *)(b + w.d_gate_up);
    float *parts = d_row_weights_dev ? (float *)(b + w.parts) : nullptr;
    const bool large = n_rows >= 192LL * g.n;
    if (n_rows > 0) {
        act_args a = {g, (const uint16_t *)dy_dev, dy_stride, (const uint16_t *)experts->down_dev, row_weights_dev, (const uint16_t *)kept_dev, act, d_act, parts, n_rows, H, I, 0};
        int n_parts = 0;
        rc = large ? launch_act<256, 256>(a, s, &n_parts) : launch_act<128, 64>(a, s, &n_parts);
        if (rc != MW_OK) return rc;
        if (parts) {
            hipLaunchKernelGGL(k_ffn_weights, dim3((uint32_t)pieces(n_rows, 256)), dim3(256), 0, s, g, parts, n_parts, d_row_weights_dev);
            MW_HIP_CHECK(hipGetLastError());
        }
        if (dx_dev) {
            rows_args d = {g, d_act, 2 * (int64_t)I, (const uint16_t *)experts->gate_up_dev, nullptr, (uint16_t *)dx_dev, dx_stride, 2 * I, H, 0};
            rc = large ? launch_rows<256, 256, true>(d, s) : launch_rows<128, 64, true>(d, s);
            if (rc != MW_OK) return rc;
        }
    }
    if (d_gate_up_dev) {
        grads_args a = {g, d_act, (const uint16_t *)x_dev, 2 * (int64_t)I, x_stride, (uint16_t *)d_gate_up_dev, 2 * I, H, 0, 0};
        rc = launch_grads<256, 256>(a, s);
        if (rc != MW_OK) return rc;
    }
    if (d_down_dev) {
        grads_args a = {g, (const uint16_t *)dy_dev, act, dy_stride, I, (uint16_t *)d_down_dev, H, I, 0, 0};
        rc = launch_grads<256, 256>(a, s);
    }
    return rc;
}
