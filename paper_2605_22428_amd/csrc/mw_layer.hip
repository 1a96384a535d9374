// mw_moe_layer: the local experts of a batch of at most 256 tokens, from gate scores (or ids and weights) to the summed output.
//
//   act[pair] = w silu(Wg x) * (Wu x)        one pair: a token and a local expert it goes to (k_layer_up)
//   out[t]    = sum over the token's pairs of Wd act[pair]                                    (k_layer_down)
//
// Every weight of an expert that a token goes to has to be read once and is used for a few tokens only, so the weights' bytes bound both
// kernels.  They are streamed from memory into registers in the layout that the matrix instruction takes, never through LDS: 16
// weight rows are one side, up to 16 tokens the other, and whichever columns have no token cost nothing that counts.
#include <float.h>

#include "mw_math.h"

namespace {

constexpr int kChunk = 128;              // columns a wave takes at a time: a scale block of fp8 weights

struct layer_args {
    const int32_t *ids;                  // [T][K]
    const float *weights;                // [T][K]
    const int32_t *eslot;                // [E] (rank << 16) | slot
    int32_t my_rank, T, K, E, L, H, I;
    const uint16_t *x; int64_t x_stride; // bf16 rows
    const void *up, *down;               // [L][2][I][H], [L][H][I]
    const float *up_scale, *down_scale;  // fp8: [L][2][ceil(I/128)][ceil(H/128)], [L][ceil(H/128)][ceil(I/128)]
    uint16_t *act_hi, *act_lo;           // [T * K][I] bf16: act rounded, and what the rounding left
    float *y;                            // [T * K][H] (batches over 16 tokens)
    uint16_t *out; int64_t out_stride;
    uint32_t *flags;                     // or null
};

__device__ __forceinline__ int local_slot(const layer_args &a, int32_t id)
{
    if (id < 0 || id >= a.E) return -1;
    const int32_t v = a.eslot[id];
    return (v >> 16) == a.my_rank ? (v & 0xffff) : -1;
}

// An expert that a token names twice is one pair: the first place's, with both weights.
__device__ __forceinline__ bool first_place(const layer_args &a, int p, int32_t id)
{
    for (int q = p - p % a.K; q < p; ++q) if (a.ids[q] == id) return false;
    return true;
}
__device__ __forceinline__ float pair_weight(const layer_args &a, int p, int32_t id)
{
    float w = 0.0f;
    for (int q = p; q < p - p % a.K + a.K; ++q) if (a.ids[q] == id) w += a.weights[q];
    return w;
}

constexpr int kWords = MW_GATE_MAX_EXPERTS / 32;
// The local experts that some token goes to, as bits; every thread of the workgroup.
__device__ __forceinline__ void hit_experts(const layer_args &a, uint32_t *bits, uint32_t *bad)
{
    for (int i = threadIdx.x; i < kWords; i += blockDim.x) bits[i] = 0;
    __syncthreads();
    bool wrong = false;
    for (int p = threadIdx.x; p < a.T * a.K; p += blockDim.x) {
        const int32_t id = a.ids[p];
        wrong |= id < -1 || id >= a.E;
        const int le = local_slot(a, id);
        if (le >= 0) atomicOr(&bits[le >> 5], 1u << (le & 31));
    }
    if (bad && wrong) atomicOr(bad, MW_FLAG_BAD_EXPERT);
    __syncthreads();
}
// The n-th of them, or -1.
__device__ __forceinline__ int nth_hit(const uint32_t *bits, int n)
{
    for (int w = 0; w < kWords; ++w) {
        uint32_t b = bits[w];
        const int c = __popc(b);
        if (n < c) {
            for (; n > 0; --n) b &= b - 1;
            return w * 32 + __ffs(b) - 1;
        }
        n -= c;
    }
    return -1;
}
// The pairs of local expert `le` (their order does not matter: a pair is a column of its own everywhere).
__device__ __forceinline__ int pairs_of(const layer_args &a, int le, int *count, uint16_t *list)
{
    if (threadIdx.x == 0) *count = 0;
    __syncthreads();
    for (int p = threadIdx.x; p < a.T * a.K; p += blockDim.x) {
        const int32_t id = a.ids[p];
        if (local_slot(a, id) == le && first_place(a, p, id)) list[atomicAdd(count, 1)] = (uint16_t)p;
    }
    __syncthreads();
    return *count;
}

// 8 weights of one lane for one matrix instruction, as bf16.  Of a span of 64 columns lane group g holds columns g * 16 .. + 15 and
// the span takes two instructions (half 0, half 1): bf16 weights are two 16-byte loads a span, fp8 weights one.
template <bool kFp8> struct span;
template <> struct span<false> {
    bf16x8 v[2];
    __device__ __forceinline__ void load(const void *row, int at, int limit)
    {
        const bf16x8 zero = {};
        const uint16_t *p = (const uint16_t *)row;
        v[0] = at < limit ? __builtin_bit_cast(bf16x8, mw_ld16((const u32x4 *)(p + at))) : zero;
        v[1] = at + 8 < limit ? __builtin_bit_cast(bf16x8, mw_ld16((const u32x4 *)(p + at + 8))) : zero;
    }
    __device__ __forceinline__ bf16x8 half(int i) const { return v[i]; }
};
template <> struct span<true> {
    u32x4 c;
    __device__ __forceinline__ void load(const void *row, int at, int limit)
    {
        const u32x4 zero = {};
        c = at < limit ? mw_ld16((const u32x4 *)((const uint8_t *)row + at)) : zero;
    }
    __device__ __forceinline__ bf16x8 half(int i) const
    {
        const uint32_t a = i ? c.z : c.x, b = i ? c.w : c.y;         // (every e4m3 value is a bf16 value)
        bf16x8 r;
        const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
        const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
        r[0] = p0[0]; r[1] = p0[1]; r[2] = p1[0]; r[3] = p1[1]; r[4] = p2[0]; r[5] = p2[1]; r[6] = p3[0]; r[7] = p3[1];
        return r;
    }
};
__device__ __forceinline__ bf16x8 load8(const uint16_t *row, int at, int limit, bool live)
{
    const bf16x8 zero = {};
    return live && at < limit ? *(const bf16x8 *)(row + at) : zero;
}
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 add_scaled(f32x4 to, f32x4 v, float s)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] += s * v[i];
    return to;
}

// grid: (16 rows of I, hit experts).  A workgroup's waves take every kUpWaves-th chunk of the columns each.
constexpr int kUpWaves = 4;
template <bool kFp8, int kTiles>
__device__ __forceinline__ void up_columns(const layer_args &a, int le, int row0, const uint16_t *list, int first, int count, float *part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const int row = min(row0 + n, a.I - 1);
    const int64_t unit = kFp8 ? 1 : 2;
    const char *gate = (const char *)a.up + (((int64_t)le * 2) * a.I + row) * a.H * unit;
    const char *up = gate + (int64_t)a.I * a.H * unit;
    const int cblocks = (a.H + 127) / 128, rblocks = (a.I + 127) / 128;
    const float *gs = kFp8 ? a.up_scale + ((int64_t)le * 2 * rblocks + row0 / 128) * cblocks : nullptr;
    const float *us = kFp8 ? gs + (int64_t)rblocks * cblocks : nullptr;
    const uint16_t *xr[kTiles];
    bool live[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        live[i] = first + i * 16 + n < count;
        xr[i] = a.x + (int64_t)(list[live[i] ? first + i * 16 + n : 0] / a.K) * a.x_stride;
    }
    f32x4 accg[kTiles] = {}, accu[kTiles] = {};
    for (int c = wave; c * kChunk < a.H; c += kUpWaves) {
        span<kFp8> wg[2], wu[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            wg[j].load(gate, c * kChunk + j * 64 + g * 16, a.H);
            wu[j].load(up, c * kChunk + j * 64 + g * 16, a.H);
        }
        f32x4 cg[kTiles] = {}, cu[kTiles] = {};
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bf16x8 ag = wg[j].half(h), au = wu[j].half(h);
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    const bf16x8 b = load8(xr[i], c * kChunk + j * 64 + g * 16 + h * 8, a.H, live[i]);
                    if constexpr (kFp8) { cg[i] = mma(ag, b, cg[i]); cu[i] = mma(au, b, cu[i]); }
                    else { accg[i] = mma(ag, b, accg[i]); accu[i] = mma(au, b, accu[i]); }
                }
            }
        if constexpr (kFp8) {
            const float sg = gs[c], su = us[c];
#pragma unroll
            for (int i = 0; i < kTiles; ++i) { accg[i] = add_scaled(accg[i], cg[i], sg); accu[i] = add_scaled(accu[i], cu[i], su); }
        }
    }
    // part [wave][gate, up][column][16 rows]
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        *(f32x4 *)&part[((wave * 2 + 0) * kTiles * 16 + i * 16 + n) * 16 + g * 4] = accg[i];
        *(f32x4 *)&part[((wave * 2 + 1) * kTiles * 16 + i * 16 + n) * 16 + g * 4] = accu[i];
    }
    __syncthreads();
    for (int o = threadIdx.x; o < kTiles * 256; o += kUpWaves * 64) {
        const int col = o >> 4, r = o & 15;
        if (first + col >= count || row0 + r >= a.I) continue;
        float vg = 0.0f, vu = 0.0f;
#pragma unroll
        for (int w = 0; w < kUpWaves; ++w) {
            vg += part[(w * 2 + 0) * kTiles * 256 + o];
            vu += part[(w * 2 + 1) * kTiles * 256 + o];
        }
        const int p = list[first + col];
        const float v = vg / (1.0f + expf(-vg)) * vu * pair_weight(a, p, a.ids[p]);
        // Kept as a sum of two bf16 values, 16 bits of mantissa: the second costs the next kernel a matrix instruction that it has to
        // spare, where one value alone would add as much error as the output's own rounding does.
        const uint16_t hi = mw_f32_to_bf16(v);
        const float rest = v - mw_bf16_to_f32(hi);
        a.act_hi[(int64_t)p * a.I + row0 + r] = hi;
        a.act_lo[(int64_t)p * a.I + row0 + r] = fabsf(v) <= FLT_MAX && rest == rest && fabsf(rest) <= FLT_MAX ? mw_f32_to_bf16(rest) : 0;
    }
    __syncthreads();
}

template <bool kFp8>
__global__ __launch_bounds__(kUpWaves * 64) void k_layer_up(layer_args a)
{
    __shared__ __align__(16) float part[kUpWaves * 2 * 4 * 256];
    __shared__ uint32_t bits[kWords];
    __shared__ uint16_t list[MW_LAYER_MAX_TOKENS];
    __shared__ int n_pairs;
    hit_experts(a, bits, blockIdx.x == 0 && blockIdx.y == 0 ? a.flags : nullptr);
    const int le = nth_hit(bits, blockIdx.y);
    if (le < 0) return;
    const int count = pairs_of(a, le, &n_pairs, list), row0 = blockIdx.x * 16;
    for (int first = 0; first < count;) {
        const int left = count - first;
        if (left <= 16) { up_columns<kFp8, 1>(a, le, row0, list, first, count, part); first += 16; }
        else if (left <= 32) { up_columns<kFp8, 2>(a, le, row0, list, first, count, part); first += 32; }
        else { up_columns<kFp8, 4>(a, le, row0, list, first, count, part); first += 64; }
    }
}

// Batches of at most 16 tokens: a token is a column, the experts' products are one long sum.  grid: 16 rows of H.
constexpr int kDownWaves = 4;
template <bool kFp8>
__global__ __launch_bounds__(kDownWaves * 64) void k_layer_down_few(layer_args a)
{
    __shared__ __align__(16) float part[kDownWaves * 256];
    __shared__ uint32_t bits[kWords];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4, row0 = blockIdx.x * 16;
    hit_experts(a, bits, nullptr);
    const int row = min(row0 + n, a.H - 1), chunks = (a.I + kChunk - 1) / kChunk, rblocks = (a.H + 127) / 128;
    f32x4 acc = {};
    int u = 0;
    for (int w = 0; w < kWords; ++w)
        for (uint32_t b = bits[w]; b; b &= b - 1) {
            const int le = w * 32 + __ffs(b) - 1;
            int pair = -1;                       // the column's token's place in the batch's list, if it goes to this expert
            if (n < a.T)
                for (int k = a.K - 1; k >= 0; --k) if (local_slot(a, a.ids[n * a.K + k]) == le) pair = n * a.K + k;
            const uint16_t *hi = a.act_hi + (int64_t)max(pair, 0) * a.I, *lo = a.act_lo + (int64_t)max(pair, 0) * a.I;
            const char *down = (const char *)a.down + ((int64_t)le * a.H + row) * a.I * (kFp8 ? 1 : 2);
            for (int c = 0; c < chunks; ++c, ++u) {
                if (u % kDownWaves != wave) continue;
                span<kFp8> wd[2];
                f32x4 cc = {};
#pragma unroll
                for (int j = 0; j < 2; ++j) wd[j].load(down, c * kChunk + j * 64 + g * 16, a.I);
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int at = c * kChunk + j * 64 + g * 16 + h * 8;
                        const bf16x8 v = wd[j].half(h);
                        cc = mma(v, load8(hi, at, a.I, pair >= 0), cc);
                        cc = mma(v, load8(lo, at, a.I, pair >= 0), cc);
                    }
                const float s = kFp8 ? a.down_scale[((int64_t)le * rblocks + row0 / 128) * chunks + c] : 1.0f;
                if (pair >= 0) acc = add_scaled(acc, cc, s);         // (0 times a weight that is no number is not 0)
            }
        }
    *(f32x4 *)&part[wave * 256 + n * 16 + g * 4] = acc;
    __syncthreads();
    const int col = threadIdx.x >> 4, r = threadIdx.x & 15;
    if (col < a.T && row0 + r < a.H) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kDownWaves; ++w) v += part[w * 256 + col * 16 + r];
        a.out[(int64_t)col * a.out_stride + row0 + r] = mw_f32_to_bf16(v);
    }
}

// Larger batches: a pair's product by itself.  grid: (16 rows of H, hit experts).
template <bool kFp8, int kTiles>
__device__ __forceinline__ void down_columns(const layer_args &a, int le, int row0, const uint16_t *list, int first, int count, float *part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const int row = min(row0 + n, a.H - 1), chunks = (a.I + kChunk - 1) / kChunk, rblocks = (a.H + 127) / 128;
    const char *down = (const char *)a.down + ((int64_t)le * a.H + row) * a.I * (kFp8 ? 1 : 2);
    const uint16_t *hi[kTiles], *lo[kTiles];
    bool live[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        live[i] = first + i * 16 + n < count;
        const int64_t p = list[live[i] ? first + i * 16 + n : 0];
        hi[i] = a.act_hi + p * a.I;
        lo[i] = a.act_lo + p * a.I;
    }
    f32x4 acc[kTiles] = {};
    for (int c = wave; c < chunks; c += kDownWaves) {
        span<kFp8> wd[2];
        f32x4 cc[kTiles] = {};
#pragma unroll
        for (int j = 0; j < 2; ++j) wd[j].load(down, c * kChunk + j * 64 + g * 16, a.I);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = c * kChunk + j * 64 + g * 16 + h * 8;
                const bf16x8 v = wd[j].half(h);
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    cc[i] = mma(v, load8(hi[i], at, a.I, live[i]), cc[i]);
                    cc[i] = mma(v, load8(lo[i], at, a.I, live[i]), cc[i]);
                }
            }
        const float s = kFp8 ? a.down_scale[((int64_t)le * rblocks + row0 / 128) * chunks + c] : 1.0f;
#pragma unroll
        for (int i = 0; i < kTiles; ++i) acc[i] = add_scaled(acc[i], cc[i], s);
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i) *(f32x4 *)&part[wave * kTiles * 256 + (i * 16 + n) * 16 + g * 4] = acc[i];
    __syncthreads();
    for (int o = threadIdx.x; o < kTiles * 256; o += kDownWaves * 64) {
        const int col = o >> 4, r = o & 15;
        if (first + col >= count || row0 + r >= a.H) continue;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kDownWaves; ++w) v += part[w * kTiles * 256 + o];
        a.y[(int64_t)list[first + col] * a.H + row0 + r] = v;
    }
    __syncthreads();
}

template <bool kFp8>
__global__ __launch_bounds__(kDownWaves * 64) void k_layer_down(layer_args a)
{
    __shared__ __align__(16) float part[kDownWaves * 4 * 256];
    __shared__ uint32_t bits[kWords];
    __shared__ uint16_t list[MW_LAYER_MAX_TOKENS];
    __shared__ int n_pairs;
    hit_experts(a, bits, nullptr);
    const int le = nth_hit(bits, blockIdx.y);
    if (le < 0) return;
    const int count = pairs_of(a, le, &n_pairs, list), row0 = blockIdx.x * 16;
    for (int first = 0; first < count;) {
        const int left = count - first;
        if (left <= 16) { down_columns<kFp8, 1>(a, le, row0, list, first, count, part); first += 16; }
        else if (left <= 32) { down_columns<kFp8, 2>(a, le, row0, list, first, count, part); first += 32; }
        else { down_columns<kFp8, 4>(a, le, row0, list, first, count, part); first += 64; }
    }
}

// out[t] = the sum of its pairs, in the order of its ids.  grid: (1024 columns, token).
__global__ __launch_bounds__(256) void k_layer_sum(layer_args a)
{
    __shared__ int use[MW_MAX_TOPK];
    const int t = blockIdx.y;
    if ((int)threadIdx.x < a.K) {
        const int p = t * a.K + threadIdx.x;
        const int32_t id = a.ids[p];
        use[threadIdx.x] = local_slot(a, id) >= 0 && first_place(a, p, id);
    }
    __syncthreads();
    const int h = (blockIdx.x * 256 + threadIdx.x) * 4;
    if (h >= a.H) return;                        // (H is a multiple of 8)
    f32x4 v = {};
    for (int k = 0; k < a.K; ++k)
        if (use[k]) v += *(const f32x4 *)&a.y[((int64_t)t * a.K + k) * a.H + h];
    bf16x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (__bf16)v[i];
    *(bf16x4 *)&a.out[(int64_t)t * a.out_stride + h] = o;
}

struct layer_ws { int64_t hi, lo, y, total; };
layer_ws layer_layout(const mw_ctx *ctx, int64_t inter, int64_t tokens)
{
    layer_ws w;
    int64_t o = 0;
    const int64_t pairs = tokens * ctx->cfg.top_k;
    w.hi = o; o += mw_align_up(2 * pairs * inter, 256);
    w.lo = o; o += mw_align_up(2 * pairs * inter, 256);
    w.y = o;  o += tokens > 16 ? mw_align_up(4 * pairs * ctx->cfg.hidden, 256) : 0;
    w.total = o > 0 ? o : 256;
    return w;
}

int32_t experts_ready(const mw_ctx *ctx, const mw_experts *e)
{
    if (!e || ctx->cfg.n_experts < 1 || e->inter < 1) return MW_ERR_INVALID_ARG;
    if (ctx->cfg.n_experts > MW_GATE_MAX_EXPERTS || ctx->cfg.row_format == MW_ROW_BYTES) return MW_ERR_UNSUPPORTED;
    const bool fp8 = e->format == MW_ROW_FP8_E4M3_BLOCK128;
    if (!fp8 && e->format != MW_ROW_BF16) return MW_ERR_INVALID_ARG;
    if (fp8 != (e->gate_up_scale_dev != nullptr) || fp8 != (e->down_scale_dev != nullptr)) return MW_ERR_INVALID_ARG;
    const int32_t unit = fp8 ? 16 : 8;           // rows of whole 16-byte pieces
    if (ctx->cfg.hidden % unit != 0 || e->inter % unit != 0 || e->inter > (1 << 20)) return MW_ERR_UNSUPPORTED;
    if (ctx->n_local > 0 && (!e->gate_up_dev || !e->down_dev)) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)e->gate_up_dev | (uintptr_t)e->down_dev) & 15u) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)e->gate_up_scale_dev | (uintptr_t)e->down_scale_dev) & 3u) return MW_ERR_INVALID_ARG;
    return MW_OK;
}

}  // namespace

extern "C" MW_API int32_t mw_moe_workspace_bytes(mw_ctx *ctx, const mw_experts *experts, int32_t max_tokens, int64_t *out_bytes)
{
    if (!ctx || !out_bytes || max_tokens < 0) return MW_ERR_INVALID_ARG;
    const int32_t rc = experts_ready(ctx, experts);
    if (rc != MW_OK) return rc;
    if (max_tokens > MW_LAYER_MAX_TOKENS) return MW_ERR_CAPACITY;
    *out_bytes = layer_layout(ctx, experts->inter, max_tokens).total;
    return MW_OK;
}

extern "C" MW_API int32_t mw_moe_layer(mw_ctx *ctx, const mw_gate *gate, const void *logits_dev, int32_t logit_format, int64_t logit_stride,
                                       const float *bias_dev, const mw_experts *experts, const void *x_dev, int64_t x_stride, int32_t n_tokens,
                                       int32_t *topk_ids_dev, float *topk_weights_dev, void *out_dev, int64_t out_stride,
                                       uint32_t *error_flags_dev, void *workspace_dev, int64_t workspace_bytes, void *stream)
{
    if (!ctx || n_tokens < 0) return MW_ERR_INVALID_ARG;
    int32_t rc = experts_ready(ctx, experts);
    if (rc == MW_OK) rc = mw_on_device_of(ctx);
    if (rc != MW_OK) return rc;
    if (n_tokens > MW_LAYER_MAX_TOKENS || n_tokens > ctx->cfg.max_tokens) return MW_ERR_CAPACITY;
    const int32_t H = ctx->cfg.hidden, I = experts->inter;
    if (x_stride < H || out_stride < H || x_stride % 8 != 0 || out_stride % 8 != 0) return MW_ERR_INVALID_ARG;
    if (((uintptr_t)x_dev | (uintptr_t)out_dev) & 15u) return MW_ERR_INVALID_ARG;
    if ((uintptr_t)error_flags_dev & 3u) return MW_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!x_dev || !topk_ids_dev || !topk_weights_dev || !out_dev)) return MW_ERR_INVALID_ARG;
    const layer_ws w = layer_layout(ctx, I, n_tokens);
    if (!workspace_dev || ((uintptr_t)workspace_dev & 255u) || workspace_bytes < w.total) return MW_ERR_WORKSPACE;
    if (logits_dev || gate) {
        rc = mw_route(ctx, gate, logits_dev, logit_format, logit_stride, bias_dev, n_tokens, topk_ids_dev, topk_weights_dev, stream);
        if (rc != MW_OK) return rc;
    }
    if (n_tokens == 0) return MW_OK;
    char *b = (char *)workspace_dev;
    layer_args a;
    a.ids = topk_ids_dev; a.weights = topk_weights_dev; a.eslot = ctx->d_eslot;
    a.my_rank = ctx->cfg.my_rank; a.T = n_tokens; a.K = ctx->cfg.top_k; a.E = ctx->cfg.n_experts; a.L = ctx->n_local; a.H = H; a.I = I;
    a.x = (const uint16_t *)x_dev; a.x_stride = x_stride;
    a.up = experts->gate_up_dev; a.down = experts->down_dev;
    a.up_scale = experts->gate_up_scale_dev; a.down_scale = experts->down_scale_dev;
    a.act_hi = (uint16_t *)(b + w.hi); a.act_lo = (uint16_t *)(b + w.lo); a.y = (float *)(b + w.y);
    a.out = (uint16_t *)out_dev; a.out_stride = out_stride;
    a.flags = error_flags_dev;
    const hipStream_t s = (hipStream_t)stream;
    const int64_t pairs = (int64_t)n_tokens * a.K;
    const uint32_t hits = (uint32_t)(a.L < 1 ? 1 : pairs < a.L ? pairs : a.L);       // experts that can be hit at most
    const dim3 up((uint32_t)((I + 15) / 16), hits), down((uint32_t)((H + 15) / 16), n_tokens <= 16 ? 1 : hits);
    const bool fp8 = experts->format == MW_ROW_FP8_E4M3_BLOCK128;
    if (fp8) hipLaunchKernelGGL((k_layer_up<true>), up, dim3(kUpWaves * 64), 0, s, a);
    else hipLaunchKernelGGL((k_layer_up<false>), up, dim3(kUpWaves * 64), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    if (n_tokens <= 16) {
        if (fp8) hipLaunchKernelGGL((k_layer_down_few<true>), down, dim3(kDownWaves * 64), 0, s, a);
        else hipLaunchKernelGGL((k_layer_down_few<false>), down, dim3(kDownWaves * 64), 0, s, a);
        MW_HIP_CHECK(hipGetLastError());
        return MW_OK;
    }
    if (fp8) hipLaunchKernelGGL((k_layer_down<true>), down, dim3(kDownWaves * 64), 0, s, a);
    else hipLaunchKernelGGL((k_layer_down<false>), down, dim3(kDownWaves * 64), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(k_layer_sum, dim3((uint32_t)((H + 1023) / 1024), (uint32_t)n_tokens), dim3(256), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
