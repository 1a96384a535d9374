// mw_quantize_rows, mw_matmul_int8: products in 8-bit integers with a scale for each row and each output channel, and the experts that use them.
#include "mw_ffn.h"
#include "mw_few.h"

namespace {

// ---- rows -> codes and scales ---------------------------------------------------------------------------------------
// code = round-half-even(127 x / a), a the row's largest |x|, of the exact quotient v.  x and a have eight significant bits, so v is a half of an odd number exactly or at least
// |v| 2^-17 away from one: |v - (2m + 1) / 2| = |254 X 2^d - (2m + 1) A| / 2A with whole X, A of eight bits and d the difference of their exponents, and a numerator that is not 0
// is 2^d at least.  y = x (127 / a) is off by |v| 2^-23 at most.  Rounded to 18 bits (off by |v| 2^-18 at most) it is such a half exactly where v is one, and on v's side of it
// elsewhere; adding 1.5 2^23 then rounds to the even whole number and leaves it in the low bits.  Six instructions a value instead of a division's dozen: 8192 rows of
// 7168 values, 176 MB, 36 -> 31 us (5.7 TB/s), 16384 rows of 2048, 100 MB, 27 -> 18 us.
struct quant_args {
    const uint16_t *x; int64_t x_stride;
    int8_t *codes; int64_t codes_stride;
    float *scales;
    int64_t n_rows;
    const int64_t *end;                     // rows from here on are left alone; or null
    int32_t n;
};
__device__ __forceinline__ uint32_t row_most(uint32_t most, u32x4 q)        // |x| as its bits, which order like the values; NaN and infinity are above all
{
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, max(q[i] << 16 & 0x7fff0000u, q[i] & 0x7fff0000u));
    return most;
}
struct row_factor { float pre, by; };                                       // pre: a power of two, so that 127 / a does not overflow
__device__ __forceinline__ row_factor factor_of(uint32_t most)
{
    const float a = __uint_as_float(most), pre = a < 0x1p-60f ? 0x1p64f : 1.0f;
    return most == 0 || most >= 0x7f800000u ? row_factor{0.0f, 0.0f} : row_factor{pre, 127.0f / (a * pre)};
}
__device__ __forceinline__ uint32_t code_of(uint32_t bits, row_factor f)    // in the low byte
{
    const float y = __uint_as_float(bits) * f.pre * f.by;
    return __float_as_uint(__uint_as_float((__float_as_uint(y) + 0x20u) & ~0x3fu) + 12582912.0f);
}
__device__ __forceinline__ void put_codes(const quant_args &a, int64_t row, int chunk, u32x4 q, row_factor f, bool some)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    u32x2 o;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t c0 = code_of(q[i * 2] << 16, f), c1 = code_of(q[i * 2] & 0xffff0000u, f), c2 = code_of(q[i * 2 + 1] << 16, f), c3 = code_of(q[i * 2 + 1] & 0xffff0000u, f);
        const uint32_t low = __builtin_amdgcn_perm(c1, c0, 0x0c0c0400u), high = __builtin_amdgcn_perm(c3, c2, 0x04000c0cu);
        o[i] = some ? low | high : 0u;
    }
    *(u32x2 *)(a.codes + row * a.codes_stride + chunk * 8) = o;
}
__device__ __forceinline__ float scale_of(uint32_t most) { return most < 0x7f800000u ? __uint_as_float(most) / 127.0f : __uint_as_float(0x7fc00000u); }

constexpr uint32_t kQuantizeRun = 1u << 20;        // workgroups along x: a grid has fewer than 2^32 threads along one axis
// kWaves waves a row; up to kChunks pieces of eight values a lane stay in registers, of longer rows the rest is read twice.
template <int kWaves, int kChunks>
__global__ __launch_bounds__(256) void k_quantize(quant_args a)
{
    __shared__ uint32_t waves[4];
    constexpr int kLanes = kWaves * 64;
    const int tid = (int)threadIdx.x % kLanes, chunks = a.n / 8;
    const int64_t row = ((int64_t)blockIdx.y * kQuantizeRun + blockIdx.x) * (4 / kWaves) + (int)threadIdx.x / kLanes;
    if (row >= a.n_rows || (a.end && row >= *a.end)) return;                // (a wave's or the workgroup's)
    const uint16_t *x = a.x + row * a.x_stride;
    u32x4 v[kChunks];
    uint32_t most = 0;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) v[c] = tid + c * kLanes < chunks ? *(const u32x4 *)(x + (tid + c * kLanes) * 8) : u32x4{};
#pragma unroll
    for (int c = 0; c < kChunks; ++c) most = row_most(most, v[c]);
    for (int c = tid + kChunks * kLanes; c < chunks; c += kLanes) most = row_most(most, *(const u32x4 *)(x + c * 8));
    most = mw_wave_max(most);
    if constexpr (kWaves > 1) {
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = most;
        mw_lds_barrier();
        most = max(max(waves[0], waves[1]), max(waves[2], waves[3]));
    }
    if (tid == 0) a.scales[row] = scale_of(most);
    const row_factor f = factor_of(most);
    const bool some = f.by != 0.0f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) if (tid + c * kLanes < chunks) put_codes(a, row, tid + c * kLanes, v[c], f, some);
    for (int c = tid + kChunks * kLanes; c < chunks; c += kLanes) put_codes(a, row, c, *(const u32x4 *)(x + c * 8), f, some);
}

// ---- rows of codes times matrices of codes ------------------------------------------------------------------------
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
// Sums of codes are whole numbers, so their order and parts change nothing; the factors come in once, in fp32, at the end.  kGated: y = silu(gate) * up, columns as in the bf16 experts'.
// Medians of 33 calls in a kernel trace (the least): 8192 rows, 7168 -> 7168, 386 us (366), 2180 TOP/s; 16384 rows of four experts 7168 x 2048, gated, 467 us (457), 2060 TOP/s, and back 276 us
// (262), 1740 (16 steps a tile).
template <int kCols, int kRows, bool kGated, bool kF32>
struct int8_op {
    static constexpr int kP = kCols, kQ = kRows;
    static constexpr bool kTrP = false, kInt8 = true, kPair = kGated, kRowValues = true;
    static constexpr int kTerms = 1;
    struct args {
        row_groups g;
        const int8_t *x; int64_t x_stride;
        const float *x_scale;
        const int8_t *w;                        // [n][N][K]; kGated: [n][2][N][K]
        const float *w_scale;                   // [n][N]; [n][2][N]
        const float *row_weights;               // or null
        void *y; int64_t y_stride;              // bf16 or fp32 rows
        float *parts;
        int32_t K, N, p_tiles;
    };
    static constexpr int kHalf = kGated ? kP / 4 : kP / 2;              // columns of half the waves
    static __device__ __forceinline__ void feeds(const args &a, const tile_at &at, tile_feed<kP, false, true> &fp, tile_feed<kQ, false, true> &fq)
    {
        const int col0 = at.p * 2 * kHalf;
        fp.rows((const char *)(a.w + ((int64_t)at.e * (kGated ? 2 : 1) * a.N + col0) * a.K), a.K, [&](int r) {
            const int in = r % (kP / 2), up = in / kHalf, col = r / (kP / 2) * kHalf + in % kHalf;
            return col0 + col < a.N ? (uint32_t)(up * a.N + col) * (uint32_t)a.K : kNowhereAt;
        });
        fq.rows((const char *)(a.x + at.first * a.x_stride), a.K, [&](int r) { return r < at.rows ? (uint32_t)r * (uint32_t)a.x_stride : kNowhereAt; });
    }
    static __device__ __forceinline__ f32x2 rows(const args &a, int64_t row) { return {a.x_scale[row], a.row_weights ? a.row_weights[row] : 1.0f}; }
    struct scales { f32x4 w[2], up[kGated ? 2 : 1]; };
    static __device__ __forceinline__ scales columns(const args &a, const tile_at &at, int column)
    {
        const int col = at.p * 2 * kHalf + column;
        scales s = {};
        if (col < a.N) {                                        // (N is a multiple of sixteen)
            const float *w = a.w_scale + (int64_t)at.e * (kGated ? 2 : 1) * a.N + col;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s.w[i] = *(const f32x4_any *)(w + i * 4);
                if constexpr (kGated) s.up[i] = *(const f32x4_any *)(w + a.N + i * 4);
            }
        }
        return s;
    }
    static __device__ __forceinline__ tile_nothing fetch(const args &, const tile_at &, int, int) { return {}; }
    static __device__ __forceinline__ void emit(const args &a, const tile_at &at, int row, int column, const int (&t)[8], const int (&u)[8], const scales &s, f32x2 of_row, tile_nothing)
    {
        const int col = at.p * 2 * kHalf + column;
        if (row >= at.rows || col >= a.N) return;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float value = (float)t[e] * of_row[0] * s.w[e / 4][e % 4];
            if constexpr (kGated) v[e] = value * tile_sigmoid(value) * ((float)u[e] * of_row[0] * s.up[e / 4][e % 4]);
            else v[e] = of_row[1] * value;
        }
        if constexpr (kF32) {
            float *y = (float *)a.y + (at.first + row) * a.y_stride + col;
            *(f32x4 *)y = f32x4{v[0], v[1], v[2], v[3]};
            *(f32x4 *)(y + 4) = f32x4{v[4], v[5], v[6], v[7]};
        } else {
            store_bf16((uint16_t *)a.y + (at.first + row) * a.y_stride + col, v);
        }
    }
    static __device__ __forceinline__ const void *few_matrix(const args &a, int e, int tile) { return a.w + ((int64_t)e * (kGated ? 2 : 1) * a.N + tile * (kGated ? 8 : 16)) * a.K; }
    static __device__ __forceinline__ const void *few_x(const args &a, int64_t row) { return a.x + row * a.x_stride; }
    static __device__ __forceinline__ uint32_t few_row(const args &a, int tile, int r)          // (N is a multiple of sixteen)
    {
        if (tile * (kGated ? 8 : 16) >= a.N) return kNowhere;
        return (uint32_t)(kGated ? (r >> 3) * a.N + (r & 7) : r) * (uint32_t)a.K;
    }
    static __device__ __forceinline__ void few_emit(const args &a, int e, int64_t row, int col, int t, int u)
    {
        if (col >= a.N) return;
        const float scale = a.x_scale[row], *w = a.w_scale + (int64_t)e * (kGated ? 2 : 1) * a.N + col, value = (float)t * scale * w[0];
        float v;
        if constexpr (kGated) v = value * tile_sigmoid(value) * ((float)u * scale * w[a.N]);
        else v = a.row_weights ? a.row_weights[row] * value : value;
        if constexpr (kF32) ((float *)a.y)[row * a.y_stride + col] = v;
        else ((uint16_t *)a.y)[row * a.y_stride + col] = mw_f32_to_bf16(v);
    }
};

template <bool kGated, bool kF32>
int32_t launch_int8(const typename int8_op<256, 256, kGated, kF32>::args &a, hipStream_t s)
{
    return launch_product<int8_op<256, 256, kGated, kF32>, int8_op<256, 128, kGated, kF32>, int8_op<128, 64, kGated, kF32>, true>(int8_form(a.g.n_rows, a.g.n, kGated ? 2 * (int64_t)a.N : a.N, a.K, a.parts != nullptr), a, a.N, s);
}
// Many rows take a wave each, few or long ones a workgroup each.  us: 16384 rows of 2048 values a workgroup / a wave 22 / 18; of 7168 values 62 / 67.
int32_t launch_quantize(const quant_args &a, hipStream_t s)
{
    auto grid = [](int64_t groups) { return dim3((uint32_t)(groups < kQuantizeRun ? groups : kQuantizeRun), (uint32_t)((groups + kQuantizeRun - 1) / kQuantizeRun)); };
    const dim3 four = grid((a.n_rows + 3) / 4);
    if (a.n_rows < 2048 || a.n > 4096) hipLaunchKernelGGL((k_quantize<4, 4>), grid(a.n_rows), dim3(256), 0, s, a);
    else if (a.n <= 2048) hipLaunchKernelGGL((k_quantize<1, 4>), four, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_quantize<1, 8>), four, dim3(256), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}

}  // namespace

int32_t mw_ffn_int8(const mw_experts *experts, int32_t hidden, const void *x, int64_t x_stride, const int64_t *offsets, int32_t n_local,
                    int64_t n_rows, const float *row_weights, void *y, int64_t y_stride, void *act, int8_t *codes, float *scales, float *parts, hipStream_t s)
{
    const int32_t I = experts->inter;
    const row_groups g = {offsets, n_rows, n_local};
    int32_t rc = launch_quantize({(const uint16_t *)x, x_stride, codes, hidden, scales, n_rows, offsets + n_local, hidden}, s);
    if (rc != MW_OK) return rc;
    rc = launch_int8<true, false>({g, codes, hidden, scales, (const int8_t *)experts->gate_up_dev, experts->gate_up_scale_dev, nullptr, act, I, parts, hidden, I, 0}, s);
    if (rc != MW_OK) return rc;
    rc = launch_quantize({(const uint16_t *)act, I, codes, I, scales, n_rows, offsets + n_local, I}, s);
    if (rc != MW_OK) return rc;
    return launch_int8<false, false>({g, codes, I, scales, (const int8_t *)experts->down_dev, experts->down_scale_dev, row_weights, y, y_stride, parts, I, hidden, 0}, s);
}

extern "C" MW_API int32_t mw_quantize_rows(const void *x_dev, int64_t x_stride, int64_t n_rows, int32_t n_cols, int8_t *codes_dev, int64_t codes_stride,
                                           float *scales_dev, void *stream)
{
    if (n_rows < 0 || n_cols < 1 || n_cols % 16 != 0) return MW_ERR_INVALID_ARG;
    if (n_cols > MW_INT8_MAX_IN) return MW_ERR_UNSUPPORTED;
    if (n_rows > MW_FFN_MAX_ROWS) return MW_ERR_CAPACITY;
    if (n_rows == 0) return MW_OK;
    if (!x_dev || !codes_dev || !scales_dev || (((uintptr_t)x_dev | (uintptr_t)codes_dev) & 15u) || ((uintptr_t)scales_dev & 3u)) return MW_ERR_INVALID_ARG;
    if (x_stride < n_cols || x_stride % 8 != 0 || codes_stride < n_cols || codes_stride % 16 != 0) return MW_ERR_INVALID_ARG;
    if (x_stride > MW_MAX_STRIDE || codes_stride > MW_MAX_STRIDE) return MW_ERR_UNSUPPORTED;
    return launch_quantize({(const uint16_t *)x_dev, x_stride, codes_dev, codes_stride, scales_dev, n_rows, nullptr, n_cols}, (hipStream_t)stream);
}

extern "C" MW_API int32_t mw_matmul_int8(const mw_matrices_int8 *matrices, const int8_t *codes_dev, int64_t codes_stride, const float *scales_dev,
                                         const int64_t *offsets_dev, int64_t n_rows, void *out_dev, int32_t out_format, int64_t out_stride, void *stream)
{
    const mw_matrices_int8 *m = matrices;
    if (!m || n_rows < 0 || m->n_matrices < 1 || m->n_in < 1 || m->n_out < 1 || m->n_in % 16 != 0 || m->n_out % 16 != 0) return MW_ERR_INVALID_ARG;
    if (out_format != MW_LOGITS_F32 && out_format != MW_LOGITS_BF16) return MW_ERR_INVALID_ARG;
    if (m->n_in > MW_INT8_MAX_IN || m->n_out > (1 << 20)) return MW_ERR_UNSUPPORTED;
    if (!m->codes_dev || !m->scale_dev || ((uintptr_t)m->codes_dev & 15u) || ((uintptr_t)m->scale_dev & 3u)) return MW_ERR_INVALID_ARG;
    if ((!offsets_dev && m->n_matrices != 1) || ((uintptr_t)offsets_dev & 7u)) return MW_ERR_INVALID_ARG;
    if (n_rows > MW_FFN_MAX_ROWS) return MW_ERR_CAPACITY;
    if (n_rows == 0) return MW_OK;
    if (!codes_dev || !scales_dev || !out_dev || (((uintptr_t)codes_dev | (uintptr_t)out_dev) & 15u) || ((uintptr_t)scales_dev & 3u)) return MW_ERR_INVALID_ARG;
    if (codes_stride < m->n_in || codes_stride % 16 != 0 || out_stride < m->n_out || out_stride % 8 != 0) return MW_ERR_INVALID_ARG;
    if (codes_stride > MW_MAX_STRIDE || out_stride > MW_MAX_STRIDE) return MW_ERR_UNSUPPORTED;
    const int8_op<256, 256, false, false>::args a = {{offsets_dev, n_rows, m->n_matrices}, codes_dev, codes_stride, scales_dev, m->codes_dev, m->scale_dev, nullptr, out_dev, out_stride,
                                                     nullptr, m->n_in, m->n_out, 0};
    typedef int8_op<256, 256, false, true>::args wide;
    return out_format == MW_LOGITS_F32 ? launch_int8<false, true>(__builtin_bit_cast(wide, a), (hipStream_t)stream) : launch_int8<false, false>(a, (hipStream_t)stream);
}
