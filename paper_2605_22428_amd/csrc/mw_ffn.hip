// mw_ffn, mw_ffn_backward: the experts of the rows that a dispatch brought.
#include <type_traits>

#include "mw_few.h"
#include "mw_ffn.h"

namespace {

// ---- h = silu(x Wg^T) * (x Wu^T) --------------------------------------------------------------------------------
// Half of a tile's columns are gate rows, half the up rows beside them: a lane then holds both values of an element, and neither product goes to memory unless it is kept.
// h is rounded to bf16 here, as the next product's matrix instructions take it: at most 2^-8 of h, as the output's own rounding is of y; two terms, as the few rows below have, would
// double that product.  Times at these kernels are medians of 33 calls in a kernel trace, the least in brackets; runs are uneven.  16384 rows of four experts 7168 x 2048, g and u kept: 812 us (778), 1180
// TFLOP/s; 512 rows 71 us (60) and a join of 6: 235 MB of weights at 3.3 TB/s, tiles of uneven runs fill three quarters of the CUs.
template <int kCols, int kRows>
struct up_op {
    static constexpr int kP = kCols, kQ = kRows;
    static constexpr bool kTrP = false, kInt8 = false, kPair = true, kRowValues = false;
    static constexpr int kTerms = 1;
    struct args {
        row_groups g;
        const uint16_t *x; int64_t x_stride;
        const uint16_t *w;                      // [n][2][I][H]
        uint16_t *h, *kept;                     // [rows][I], a few rows: [rows][2][I] with what its rounding left; [rows][2][I] or null
        float *parts;
        int32_t K, I, p_tiles;
    };
    static __device__ __forceinline__ void feeds(const args &a, const tile_at &at, tile_feed<kP, false, false> &fp, tile_feed<kQ, false, false> &fq)
    {
        const int col0 = at.p * (kP / 2);
        fp.rows((const char *)(a.w + ((int64_t)at.e * 2 * a.I + col0) * a.K), a.K, [&](int r) {
            const int in = r % (kP / 2), up = in / (kP / 4), col = r / (kP / 2) * (kP / 4) + in % (kP / 4);
            return col0 + col < a.I ? (uint32_t)(up * a.I + col) * (uint32_t)a.K * 2 : kNowhereAt;
        });
        fq.rows((const char *)(a.x + at.first * a.x_stride), a.K, [&](int r) { return r < at.rows ? (uint32_t)r * (uint32_t)a.x_stride * 2 : kNowhereAt; });
    }
    static __device__ __forceinline__ tile_nothing columns(const args &, const tile_at &, int) { return {}; }
    static __device__ __forceinline__ tile_nothing fetch(const args &, const tile_at &, int, int) { return {}; }
    static __device__ __forceinline__ void emit(const args &a, const tile_at &at, int row, int column, const float (&gate)[8], const float (&up)[8], tile_nothing, f32x2, tile_nothing)
    {
        const int col = at.p * (kP / 2) + column;
        if (row >= at.rows || col >= a.I) return;               // (I is a multiple of eight)
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = gate[e] * tile_sigmoid(gate[e]) * up[e];
        store_bf16(a.h + (at.first + row) * a.I + col, v);
        if (a.kept) {
            uint16_t *kept = a.kept + (at.first + row) * 2 * a.I + col;
            store_bf16<true>(kept, gate);
            store_bf16<true>(kept + a.I, up);
        }
    }
    // A few rows: eight gate rows and the eight up rows beside them.
    static __device__ __forceinline__ const void *few_matrix(const args &a, int e, int tile) { return a.w + ((int64_t)e * 2 * a.I + tile * 8) * a.K; }
    static __device__ __forceinline__ const void *few_x(const args &a, int64_t row) { return a.x + row * a.x_stride; }
    static __device__ __forceinline__ uint32_t few_row(const args &a, int tile, int r)          // (I is a multiple of eight)
    {
        if (tile * 8 >= a.I) return kNowhere;
        return (uint32_t)((r >> 3) * a.I + (r & 7)) * (uint32_t)a.K * 2;
    }
    static __device__ __forceinline__ void few_emit(const args &a, int, int64_t row, int col, float gate, float up)
    {
        if (col >= a.I) return;
        // Matrices bound these products, so h can be held as two bf16 values, 16 bits of mantissa: one alone adds as much error as the output's own rounding.
        const float v = gate * tile_sigmoid(gate) * up;
        const uint16_t high = mw_f32_to_bf16(v);
        const float rest = v - mw_bf16_to_f32(high);
        a.h[row * 2 * a.I + col] = high;
        a.h[row * 2 * a.I + a.I + col] = rest - rest == 0.0f ? mw_f32_to_bf16(rest) : 0;
        if (a.kept) {
            a.kept[row * 2 * a.I + col] = mw_f32_to_bf16(gate);
            a.kept[row * 2 * a.I + a.I + col] = mw_f32_to_bf16(up);
        }
    }
};

// ---- rows times a matrix: y = w h Wd^T, dx = [dg du] [Wg; Wu] ---------------------------------------------------
// dx: the matrices' rows are lines that the sum runs across, so both halves of gate_up are one matrix of 2 I lines, read as it lies.  16384 rows of four experts 7168 x 2048: y 460 us (432),
// 1050 TFLOP/s (sums of 2048 are 32 steps between first loads and results), dx 841 us (827), 1140.
// y and dx are stored past the caches, though what follows reads them: the call gains what its reader loses.  us, past / through them, the call, and with a copy of y or dx behind it:
// mw_ffn, 512 rows of four experts 7168 x 2048 120.0 / 120.3, 123.6 / 123.0; 2048 of eight 4096 x 1024 94.9 / 97.2, 101.6 / 102.1; 16384 of four 7168 x 2048 1223 / 1236, 1287 / 1301; dx of
// 2048 rows of eight 4096 x 1024 97.6 / 98.7, 103.3 / 103.9.
template <int kP>
__device__ __forceinline__ void columns_from(tile_feed<kP, true, false> &fp, const uint16_t *w, int col0, int K, int N)
{
    fp.lines((const char *)(w + col0), K, (int64_t)N * 2, N - col0);
}
template <int kP>
__device__ __forceinline__ void columns_from(tile_feed<kP, false, false> &fp, const uint16_t *w, int col0, int K, int N)
{
    fp.rows((const char *)(w + (int64_t)col0 * K), K, [&](int r) {
        return col0 + r < N ? (uint32_t)r * (uint32_t)K * 2 : kNowhereAt;
    });
}
template <int kCols, int kRows, bool kTr>
struct rows_op {
    static constexpr int kP = kCols, kQ = kRows;
    static constexpr int kTerms = 2;
    static constexpr bool kTrP = kTr, kInt8 = false, kPair = false, kRowValues = !kTr;          // (gradients of rows have no weights)
    struct args {
        row_groups g;
        const uint16_t *x; int64_t x_stride;    // [rows][K]
        const uint16_t *w;                      // [n][N][K], kTr: [n][K][N]
        const float *row_weights;               // or null
        uint16_t *y; int64_t y_stride;
        float *parts;
        int32_t K, N, p_tiles;
    };
    static __device__ __forceinline__ void feeds(const args &a, const tile_at &at, tile_feed<kP, kTr, false> &fp, tile_feed<kQ, false, false> &fq)
    {
        columns_from(fp, a.w + (int64_t)at.e * a.N * a.K, at.p * kP, a.K, a.N);
        fq.rows((const char *)(a.x + at.first * a.x_stride), a.K, [&](int r) { return r < at.rows ? (uint32_t)r * (uint32_t)a.x_stride * 2 : kNowhereAt; });
    }
    static __device__ __forceinline__ f32x2 rows(const args &a, int64_t row) { return {a.row_weights ? a.row_weights[row] : 1.0f, 0.0f}; }
    static __device__ __forceinline__ tile_nothing columns(const args &, const tile_at &, int) { return {}; }
    static __device__ __forceinline__ tile_nothing fetch(const args &, const tile_at &, int, int) { return {}; }
    static __device__ __forceinline__ void emit(const args &a, const tile_at &at, int row, int column, const float (&t)[8], const float (&)[8], tile_nothing, f32x2 weight, tile_nothing)
    {
        const int col = at.p * kP + column;
        if (row >= at.rows || col >= a.N) return;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = kRowValues ? weight[0] * t[e] : t[e];
        store_bf16<true>(a.y + (at.first + row) * a.y_stride + col, v);
    }
    static __device__ __forceinline__ const void *few_matrix(const args &a, int e, int tile) { return a.w + ((int64_t)e * a.N + tile * 16) * a.K; }
    static __device__ __forceinline__ const void *few_x(const args &a, int64_t row) { return a.x + row * a.x_stride; }
    static __device__ __forceinline__ uint32_t few_row(const args &a, int tile, int r)
    {
        return tile * 16 + r < a.N ? (uint32_t)r * (uint32_t)a.K * 2 : kNowhere;
    }
    static __device__ __forceinline__ void few_emit(const args &a, int, int64_t row, int col, float v, float)
    {
        if (col < a.N) a.y[row * a.y_stride + col] = mw_f32_to_bf16(a.row_weights ? a.row_weights[row] * v : v);
    }
};

// ---- da = dy Wd, and what follows from it element by element ------------------------------------------------------
// da stays in registers: g and u come beside it, and w h, dg and du leave, rounded to bf16 as operands of the products that follow (they are the products' other factors as bf16 dy and x are).
// dw's sums take da and h unrounded.  16384 rows of four experts 7168 x 2048: 451 us (438) and a join of 13, 1070 TFLOP/s, with 134 MB read and 201 MB written beside the product.
constexpr int kSum = 64;                        // columns whose da h a row sums up in the tile
template <int kCols, int kRows>
struct act_op {
    static constexpr int kP = kCols, kQ = kRows;
    static constexpr bool kTrP = true, kInt8 = false, kPair = false, kRowValues = true;
    struct args {
        row_groups g;
        const uint16_t *dy; int64_t dy_stride;
        const uint16_t *down;                   // [n][H][I]
        const float *row_weights;               // or null
        const uint16_t *kept;                   // [rows][2][I]
        uint16_t *act, *d_gate_up;              // [rows][I], [rows][2][I]
        float *sums;                            // [ceil(I / kSum)][rows] or null: sums of da h over kSum columns
        float *parts;
        int32_t K, I, p_tiles;
    };
    static __device__ __forceinline__ void feeds(const args &a, const tile_at &at, tile_feed<kP, true, false> &fp, tile_feed<kQ, false, false> &fq)
    {
        fp.lines((const char *)(a.down + (int64_t)at.e * a.K * a.I + at.p * kP), a.K, (int64_t)a.I * 2, a.I - at.p * kP);
        fq.rows((const char *)(a.dy + at.first * a.dy_stride), a.K, [&](int r) { return r < at.rows ? (uint32_t)r * (uint32_t)a.dy_stride * 2 : kNowhereAt; });
    }
    static __device__ __forceinline__ f32x2 rows(const args &a, int64_t row) { return {a.row_weights ? a.row_weights[row] : 1.0f, 0.0f}; }
    struct values { bf16x8 gate, up; };
    static __device__ __forceinline__ tile_nothing columns(const args &, const tile_at &, int) { return {}; }
    static __device__ __forceinline__ values fetch(const args &a, const tile_at &at, int row, int column)
    {
        const int col = at.p * kP + column;
        if (row >= at.rows || col >= a.I) return values{};
        const uint16_t *kept = a.kept + (at.first + row) * 2 * a.I + col;
        return values{*(const bf16x8 *)kept, *(const bf16x8 *)(kept + a.I)};
    }
    static __device__ __forceinline__ void emit(const args &a, const tile_at &at, int row, int column, const float (&da)[8], const float (&)[8], tile_nothing, f32x2 weight, const values &kept)
    {
        const int col = at.p * kP + column;
        const bool mine = row < at.rows && col < a.I;
        float sum = 0.0f;
        if (mine) {
            uint16_t *act = a.act + (at.first + row) * a.I + col, *d = a.d_gate_up + (at.first + row) * 2 * a.I + col;
            float h[8], dg[8], du[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = (float)kept.gate[e], u = (float)kept.up[e], sig = tile_sigmoid(g), silu = g * sig, dh = weight[0] * da[e];
                sum += da[e] * silu * u;
                h[e] = weight[0] * silu * u;
                dg[e] = dh * u * (sig + silu * (1.0f - sig));
                du[e] = dh * silu;
            }
            store_bf16(act, h);
            store_bf16(d, dg);
            store_bf16(d + a.I, du);
        }
        if (a.sums) {                                           // over the lanes that have kSum columns of the row: a fixed order
#pragma unroll
            for (int n = 1; n < kSum / 8; n *= 2) sum += __shfl_xor(sum, n);
            if (mine && column % kSum == 0) a.sums[(int64_t)(col / kSum) * a.g.n_rows + at.first + row] = sum;
        }
    }
};
// d_row_weights: a row's sums, sixteen rows a workgroup; sixteen lanes' sums of every sixteenth each, then of these, in a fixed order.
struct weights_args { const float *sums; float *out; int32_t n; };
__device__ __forceinline__ void row_weights_of(const row_groups &g, const weights_args &a, uint32_t block, float (*part)[17])
{
    const int r = threadIdx.x & 15, n = threadIdx.x >> 4;
    const int64_t row = (int64_t)block * 16 + r;
    const bool mine = row >= max(g.offsets[0], (int64_t)0) && row < min(g.offsets[g.n], g.n_rows);          // (no expert's rows are left alone)
    float v = 0.0f;
    if (mine) {
#pragma unroll 4
        for (int i = n; i < a.n; i += 16) v += a.sums[(int64_t)i * g.n_rows + row];
    }
    part[n][r] = v;
    __syncthreads();
    if (n > 0 || !mine) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += part[i][r];
    a.out[row] = v;
}
__global__ __launch_bounds__(256) void k_ffn_weights(row_groups g, weights_args a)
{
    __shared__ float part[16][17];
    row_weights_of(g, a, blockIdx.x, part);
}

// ---- gradients of matrices: out[q][p] = sum over a run's rows of q's value times p's ---------------------------------
struct grads_matrix {
    const uint16_t *q, *p; int64_t q_stride, p_stride;
    uint16_t *out;                          // [n][M][N], or null
    int32_t M, N, p_tiles, q_tiles;
};
struct grads_args { row_groups g; grads_matrix m[2]; uint32_t first, weights; weights_args w; };          // workgroups of m[0]; of the rows' weights, before all others
// Tiles of a matrix take as long as its run is: the XCDs get an eighth of every matrix's tiles each, and those of the longest run first.  Both matrices are one launch, and the gate weights'
// sums, which wait for the same kernel, its first workgroups.  Results are written past the caches: no one reads them soon.  16384 rows of four experts 7168 x 2048: 1162 us (1118), 1240 TFLOP/s;
// 2048 rows of eight 4096 x 1024: 85 us (80), behind the call's other products 96 (86), for 52 GFLOP and 201 MB written (writing zeros takes 28).
template <int kP, int kQ>
__global__ __launch_bounds__(kTileThreads, kP * kQ > 128 * 128 ? 1 : 5) void k_ffn_grads(grads_args a)
{
    typedef std::conditional_t<(kP * kQ > 128 * 128), tile_product<kP, kQ, true, true, false>, tile_product_short<kP, kQ, true, true, false>> product;
    typedef tile_out_bf16<kP, kQ> out_form;
    __shared__ __attribute__((aligned(1024))) char lds[product::kLds > kTileWaves * out_form::kBytes ? product::kLds : kTileWaves * out_form::kBytes];
    const uint32_t workgroup = workgroup_id();
    if (workgroup < a.weights) {
        row_weights_of(a.g, a.w, workgroup, (float (*)[17])lds);
        return;
    }
    const bool second = workgroup - a.weights >= a.first;
    const grads_matrix m = second ? a.m[1] : a.m[0];
    const uint32_t id = workgroup - a.weights - (second ? a.first : 0), each = (uint32_t)m.p_tiles * (uint32_t)m.q_tiles, per = (each + 7) / 8, at = id >> 3;
    const uint32_t tile = (id & 7) * per + at % per;
    int e = (int)(at / per);
    if (tile >= each || e >= a.g.n) return;
    int64_t first, end;
    if (a.g.n <= 64) {
        const int lane = threadIdx.x & 63;
        int64_t f = 0, l = 0;
        if (lane < a.g.n) group_bounds(a.g, lane, f, l);
        const int mine = lane < a.g.n ? (int)(l - f) : -1;
        int place = 0;
        for (int n = 0; n < a.g.n; ++n) {
            const int other = __builtin_amdgcn_readlane(mine, n);
            place += other > mine || (other == mine && n < lane);
        }
        e = __ffsll((unsigned long long)__ballot(lane < a.g.n && place == e)) - 1;
    }
    group_bounds(a.g, e, first, end);
    uint32_t pt, qt;
    tile_in_block(tile, m.p_tiles, m.q_tiles, pt, qt);
    const int q0 = (int)qt * kQ, p0 = (int)pt * kP, rows = (int)(end - first);
    tile_feed<kP, true, false> fp;
    tile_feed<kQ, true, false> fq;
    fp.lines((const char *)(m.p + first * m.p_stride + p0), rows, m.p_stride * 2, m.N - p0);
    fq.lines((const char *)(m.q + first * m.q_stride + q0), rows, m.q_stride * 2, m.M - q0);
    product t;
    t.run(fp, fq, (rows + 63) / 64, (lds_char *)lds);
    uint16_t *out = m.out + (int64_t)e * m.M * m.N;
    tile_results_bf16<kP, kQ>(t, (lds_char *)lds, [&](int row, int column, u32x4 v) {
        if (q0 + row < m.M && p0 + column < m.N) __builtin_nontemporal_store(v, (u32x4 *)(out + (int64_t)(q0 + row) * m.N + p0 + column));
    });
}

// ---- entry points -----------------------------------------------------------------------------------------------------
constexpr int64_t kPartsBytes = 256LL * 256 * 256 * 4;          // sums of a round of the large tiles; the others take less
int64_t pieces(int64_t n, int64_t each) { return (n + each - 1) / each; }

struct ffn_ws { int64_t act, d_gate_up, sums, parts, codes, scales, total; };
ffn_ws ffn_layout(const mw_experts *e, int32_t hidden, int64_t rows, bool backward)
{
    ffn_ws w = {};
    int64_t o = 0;
    auto take = [&](int64_t bytes) { const int64_t at = o; o += mw_align_up(bytes, 256); return at; };
    w.act = take((backward || e->format != MW_ROW_BF16 ? 2 : 4) * rows * e->inter);         // (a few rows' are held as two values each)
    if (backward) {
        w.d_gate_up = take(4 * rows * e->inter);
        w.sums = take(4 * rows * pieces(e->inter, kSum));
    }
    if (e->format == MW_WEIGHT_INT8_CHANNEL) {
        w.codes = take(rows * (hidden > e->inter ? hidden : e->inter));
        w.scales = take(4 * rows);
    }
    if (rows > 0) w.parts = take(kPartsBytes);
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
int32_t launch_grads(grads_args a, hipStream_t s)
{
    int64_t grid[2];
    for (int i = 0; i < 2; ++i) {
        grads_matrix &m = a.m[i];
        m.p_tiles = (int32_t)pieces(m.N, kP);
        m.q_tiles = (int32_t)pieces(m.M, kQ);
        grid[i] = m.out ? pieces((int64_t)m.p_tiles * m.q_tiles, 8) * 8 * a.g.n : 0;
    }
    const int64_t weights = a.w.out ? pieces(a.g.n_rows, 16 * 8) * 8 : 0;          // (eights, as the others are dealt out)
    if (weights + grid[0] + grid[1] > 0x7ffffff0LL) return MW_ERR_UNSUPPORTED;
    a.first = (uint32_t)grid[0];
    a.weights = (uint32_t)weights;
    hipLaunchKernelGGL((k_ffn_grads<kP, kQ>), grid_of((uint32_t)(weights + grid[0] + grid[1])), dim3(kTileThreads), 0, s, a);
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
    if (int8) return mw_ffn_int8(experts, H, x_dev, x_stride, expert_offsets_dev, ctx->n_local, n_rows, row_weights_dev, y_dev, y_stride, b + w.act, (int8_t *)(b + w.codes), (float *)(b + w.scales), (float *)(b + w.parts), s);
    const two_forms form = forward_forms(n_rows, g.n, H, I);
    const up_op<256, 256>::args u = {g, (const uint16_t *)x_dev, x_stride, (const uint16_t *)experts->gate_up_dev, (uint16_t *)(b + w.act), (uint16_t *)kept_dev, (float *)(b + w.parts), H, I, 0};
    const rows_op<256, 256, false>::args d = {g, (const uint16_t *)(b + w.act), form.second == kFew ? 2 * (int64_t)I : I, (const uint16_t *)experts->down_dev, row_weights_dev, (uint16_t *)y_dev, y_stride, (float *)(b + w.parts), I, H, 0};
    rc = launch_product<up_op<256, 256>, up_op<256, 128>, up_op<128, 64>, true>(form.first, u, I, s);
    if (rc == MW_OK) rc = launch_product<rows_op<256, 256, false>, rows_op<256, 128, false>, rows_op<128, 64, false>, true>(form.second, d, H, s);
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
    float *sums = d_row_weights_dev ? (float *)(b + w.sums) : nullptr, *parts = (float *)(b + w.parts);
    const bool matrices = d_gate_up_dev || d_down_dev;
    const weights_args of_rows = {sums, d_row_weights_dev, (int32_t)pieces(I, kSum)};
    if (n_rows > 0) {
        const two_forms form = backward_forms(n_rows, g.n, H, I);
        const act_op<256, 256>::args a = {g, (const uint16_t *)dy_dev, dy_stride, (const uint16_t *)experts->down_dev, row_weights_dev, (const uint16_t *)kept_dev, act, d_act, sums, parts, H, I, 0};
        rc = launch_product<act_op<256, 256>, act_op<256, 128>, act_op<128, 64>, false>(form.first, a, I, s);
        if (rc != MW_OK) return rc;
        if (sums && !matrices) {
            hipLaunchKernelGGL(k_ffn_weights, dim3((uint32_t)pieces(n_rows, 16)), dim3(256), 0, s, g, of_rows);
            MW_HIP_CHECK(hipGetLastError());
        }
        if (dx_dev) {
            const rows_op<256, 256, true>::args d = {g, d_act, 2 * (int64_t)I, (const uint16_t *)experts->gate_up_dev, nullptr, (uint16_t *)dx_dev, dx_stride, parts, 2 * I, H, 0};
            rc = launch_product<rows_op<256, 256, true>, rows_op<256, 128, true>, rows_op<128, 64, true>, false>(form.second, d, H, s);
            if (rc != MW_OK) return rc;
        }
    }
    if (matrices) {
        const grads_args a = {g, {{d_act, (const uint16_t *)x_dev, 2 * (int64_t)I, x_stride, (uint16_t *)d_gate_up_dev, 2 * I, H, 0, 0},
                                  {(const uint16_t *)dy_dev, act, dy_stride, I, (uint16_t *)d_down_dev, H, I, 0, 0}}, 0, 0, of_rows};
        rc = grads_large(n_rows, g.n, H, I) ? launch_grads<256, 256>(a, s) : launch_grads<128, 128>(a, s);
    }
    return rc;
}
