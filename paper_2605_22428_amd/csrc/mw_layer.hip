// mw_moe_layer: the local experts of a batch of at most 256 tokens, from gate scores (or ids and weights) to the summed output.
//
//   act[pair] = w silu(Wg x) * (Wu x)        one pair: a token and a local expert it goes to (k_layer_up)
//   out[t]    = sum over the token's pairs of Wd act[pair]                                    (k_layer_down)
//
// Every weight of an expert that a token goes to has to be read once and is used for a few tokens only, so the weights' bytes bound both
// kernels.  16 weight rows are one side of the matrix instruction and up to 16 tokens the other; whichever columns have no token cost nothing
// that counts.  Measured on one MI355X (weights of hidden 7168, inter 2048): 256 tokens of 256 experts, 32 bf16 ones here (2.8 GB):
// k_layer_up 295 us, 6.4 TB/s, k_layer_down 173 us, 5.4 TB/s, the layer 467 to 473 us, 6.0 TB/s (a plain copy: 6.8).  64 tokens, four fp8 experts
// (155 MB): 44 to 50 us; k_layer_up 22 us, 4.8 TB/s, k_layer_down 15 us, 3.4 TB/s, launches and their first round trips the rest.  One
// token, eight of 64 experts of 4096 x 1024 (201 MB): 26 us, 5.2 TB/s, and 16 us, 4.2 TB/s, the layer 45 us.  With many tokens an expert the
// tokens' way through LDS, once for every 16 or 32 rows, takes longer than the weights: 256 tokens of 8 experts, top-2, 4096 x 2048 (403 MB) 180 us.
#include "mw_stream.h"

namespace {

struct layer_args {
    const int32_t *ids;                  // [T][K]
    const float *weights;                // [T][K]
    const int32_t *eslot;                // [E] (rank << 16) | slot
    int32_t my_rank, T, K, E, L, H, I;
    const uint16_t *x; int64_t x_stride; // bf16 rows
    const void *up, *down;               // [L][2][I][H], [L][H][I]
    const float *up_scale, *down_scale;  // fp8: [L][2][ceil(I/128)][ceil(H/128)], [L][ceil(H/128)][ceil(I/128)]
    uint16_t *act_hi, *act_lo;           // [T * K][I] bf16, act_stride apart: act rounded, and what the rounding left
    int64_t act_stride;
    float *y;                            // [T * K][H] (batches over 16 tokens)
    uint16_t *out; int64_t out_stride;
    uint32_t *flags;                     // or null
};

// Slot of an id's expert among this rank's, or -1; `eslot`: the table, wherever it is.
__device__ __forceinline__ int local_slot(const layer_args &a, const int32_t *eslot, int32_t id)
{
    if (id < 0 || id >= a.E) return -1;
    const int32_t v = eslot[id];
    return (v >> 16) == a.my_rank ? (v & 0xffff) : -1;
}

// ---- which experts a batch goes to: every workgroup finds out for itself --------------------------------
constexpr int kWords = MW_GATE_MAX_EXPERTS / 32;
extern __shared__ int16_t le_of[];       // [T * K] a pair's local expert, -1: none
struct hit_set {
    uint32_t bits[kWords], before[kWords];      // experts that some token goes to; how many are in the words before
    int32_t eslot[MW_GATE_MAX_EXPERTS];
};

// Every thread of the workgroup.  The ids and the table of slots are requested together: one round trip to memory.
__device__ __forceinline__ void find_hits(const layer_args &a, hit_set &h, uint32_t *flags)
{
    constexpr int kIds = 8, kSlots = 4;
    const int tid = threadIdx.x, step = blockDim.x, pairs = a.T * a.K;
    int32_t id[kIds], slot[kSlots];
#pragma unroll
    for (int i = 0; i < kIds; ++i) id[i] = tid + i * step < pairs ? a.ids[tid + i * step] : -1;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) slot[i] = tid + i * step < a.E ? a.eslot[tid + i * step] : 0;
    if (tid < kWords) h.bits[tid] = 0;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) if (tid + i * step < a.E) h.eslot[tid + i * step] = slot[i];
    mw_lds_barrier();
    bool wrong = false;
    auto take = [&](int p, int32_t e) {
        wrong |= e < -1 || e >= a.E;
        const int le = local_slot(a, h.eslot, e);
        le_of[p] = (int16_t)le;
        if (le >= 0) atomicOr(&h.bits[le >> 5], 1u << (le & 31));
    };
#pragma unroll
    for (int i = 0; i < kIds; ++i) if (tid + i * step < pairs) take(tid + i * step, id[i]);
    for (int p = tid + kIds * step; p < pairs; p += step) take(p, a.ids[p]);
    if (flags && wrong) atomicOr(flags, MW_FLAG_BAD_EXPERT);
    mw_lds_barrier();
    if (tid < 64) {
        const uint32_t c = tid < kWords ? (uint32_t)__popc(h.bits[tid]) : 0u;
        const uint32_t incl = mw_wave_incl_scan(c);
        if (tid < kWords) h.before[tid] = incl - c;
    }
    mw_lds_barrier();
}
__device__ __forceinline__ int n_hits(const hit_set &h) { return (int)(h.before[kWords - 1] + (uint32_t)__popc(h.bits[kWords - 1])); }
__device__ __forceinline__ int index_of(const hit_set &h, int le)
{
    return (int)(h.before[le >> 5] + (uint32_t)__popc(h.bits[le >> 5] & ((1u << (le & 31)) - 1)));
}
// The n-th expert hit, n < n_hits.
__device__ __forceinline__ int nth_hit(const hit_set &h, int n)
{
    int w = 0;
    for (int i = 1; i < kWords; ++i) w = (int)h.before[i] <= n ? i : w;
    uint32_t b = h.bits[w];
    for (n -= (int)h.before[w]; n > 0; --n) b &= b - 1;
    return __builtin_amdgcn_readfirstlane(w * 32 + __ffs(b) - 1);
}
// An expert that a token names twice is one pair: the first place's, with both weights.
__device__ __forceinline__ bool first_place(const layer_args &a, int p)
{
    for (int q = p - p % a.K; q < p; ++q) if (le_of[q] == le_of[p]) return false;
    return true;
}
__device__ __forceinline__ float pair_weight(const layer_args &a, int p)
{
    float w = 0.0f;
    for (int q = p; q < p - p % a.K + a.K; ++q) if (le_of[q] == le_of[p]) w += a.weights[q];
    return w;
}
// The pairs of local expert `le` (their order does not matter: a pair is a column of its own everywhere).
__device__ __forceinline__ int pairs_of(const layer_args &a, int le, int *count, uint16_t *list)
{
    if (threadIdx.x == 0) *count = 0;
    mw_lds_barrier();
    for (int p = threadIdx.x; p < a.T * a.K; p += blockDim.x)
        if (le_of[p] == le && first_place(a, p)) list[atomicAdd(count, 1)] = (uint16_t)p;
    mw_lds_barrier();
    return __builtin_amdgcn_readfirstlane(*count);
}

// ---- act = w silu(gate) * up --------------------------------------------------------------------------------
// grid: (16 rows of I, hit experts)
constexpr int kUpWaves = 4;
template <bool kFp8, int kCols, int kHalves, int kDepth>
__device__ __forceinline__ void up_columns(const layer_args &a, int le, int row0, const uint16_t *list, int first, int count, char *lds)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), n = lane & 15, g = lane >> 4;
    const int64_t unit = kFp8 ? 1 : 2;
    const int cblocks = (a.H + 127) / 128, rblocks = (a.I + 127) / 128, l8 = lane >> 3;
    const uint32_t piece = (uint32_t)(lane & 7) * 16;
    float *part = (float *)lds;
    operands<kFp8, 2, kCols, kHalves, 1> o;
    o.w = array_at((const char *)a.up + (int64_t)le * 2 * a.I * a.H * unit);
    o.scale = array_at(kFp8 ? a.up_scale + (int64_t)le * 2 * rblocks * cblocks : nullptr);
    o.b[0] = array_at(a.x);
    o.limit = a.H;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int i = 0; i < 2; ++i) o.row[r][i] = (uint32_t)((r * a.I + min(row0 + i * 8 + l8, a.I - 1)) * unit * a.H) + piece;
        o.block[r] = (uint32_t)((r * rblocks + row0 / 128) * cblocks) * 4;
    }
#pragma unroll
    for (int c = 0; c < kCols; ++c)          // (a column without a pair repeats the first one's; its sums are not used)
#pragma unroll
        for (int i = 0; i < kHalves; ++i) {
            const int at = first + c * 16 + i * 8 + l8;
            o.col[c][0][i] = (uint32_t)((list[at < count ? at : first] / a.K) * a.x_stride * 2) + piece;
        }
    f32x4 acc[2][kCols] = {};
    stream<kFp8, 2, kCols, kHalves, 1, kUpWaves, kDepth>(o, wave, lane, lds + wave * kWaveLds<2>, acc);
    __syncthreads();                         // (the partial sums take the place of the waves' pieces)
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        // part [wave][gate, up][column][16 rows]
#pragma unroll
        for (int r = 0; r < 2; ++r) *(f32x4 *)&part[((wave * 2 + r) * 16 + n) * 16 + g * 4] = acc[r][c];
        __syncthreads();
        const int col = threadIdx.x >> 4, r = threadIdx.x & 15;
        if (threadIdx.x < 256 && first + c * 16 + col < count && row0 + r < a.I) {
            float vg = 0.0f, vu = 0.0f;
#pragma unroll
            for (int w = 0; w < kUpWaves; ++w) {
                vg += part[(w * 2 + 0) * 256 + threadIdx.x];
                vu += part[(w * 2 + 1) * 256 + threadIdx.x];
            }
            const int p = list[first + c * 16 + col];
            const float v = vg / (1.0f + expf(-vg)) * vu * pair_weight(a, p);
            // Kept as a sum of two bf16 values, 16 bits of mantissa: the second costs the next kernel a matrix instruction that it has to
            // spare, where one value alone would add as much error as the output's own rounding does.
            const uint16_t hi = mw_f32_to_bf16(v);
            const float rest = v - mw_bf16_to_f32(hi);
            a.act_hi[(int64_t)p * a.act_stride + row0 + r] = hi;
            a.act_lo[(int64_t)p * a.act_stride + row0 + r] = rest - rest == 0.0f ? mw_f32_to_bf16(rest) : 0;
        }
        __syncthreads();
    }
}

template <bool kFp8, bool kWide>
__global__ __launch_bounds__(kUpWaves * 64) void k_layer_up(layer_args a)
{
    __shared__ __align__(16) char part[kUpWaves * kWaveLds<2>];
    __shared__ hit_set hits;
    __shared__ uint16_t list[MW_LAYER_MAX_TOKENS];
    __shared__ int n_pairs;
    find_hits(a, hits, blockIdx.x == 0 && blockIdx.y == 0 ? a.flags : nullptr);
    if ((int)blockIdx.y >= n_hits(hits)) return;
    const int le = nth_hit(hits, blockIdx.y), count = pairs_of(a, le, &n_pairs, list), row0 = blockIdx.x * 16;
    for (int first = 0; first < count;) {
        const int left = count - first;
        if (left <= 8) { up_columns<kFp8, 1, 1, 3>(a, le, row0, list, first, count, part); first += 16; }
        else if (left <= 16) { up_columns<kFp8, 1, 2, 3>(a, le, row0, list, first, count, part); first += 16; }
        else if (!kWide || left <= 32) { up_columns<kFp8, 2, 2, 2>(a, le, row0, list, first, count, part); first += 32; }
        else if constexpr (kWide) { up_columns<kFp8, 4, 2, 2>(a, le, row0, list, first, count, part); first += 64; }
    }
}

// ---- out = sum of down act ------------------------------------------------------------------------------------
// Batches of at most 16 tokens: a token is a column, the experts' products are one long sum.  grid: 16 rows of H.
constexpr int kFewWaves = 8, kFewDepth = 4;
template <bool kFp8>
__global__ __launch_bounds__(kFewWaves * 64) void k_layer_down_few(layer_args a)
{
    __shared__ __align__(16) char lds[kFewWaves * kWaveLds<1>];
    __shared__ hit_set hits;
    int16_t *pair = le_of + (a.T * a.K + 7) / 8 * 8;          // [hit expert][16] the token's pair, -1: it does not go there
    uint16_t *expert = (uint16_t *)(pair + min(a.T * a.K, a.L) * 16);      // [hit expert]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), n = lane & 15, g = lane >> 4, row0 = blockIdx.x * 16;
    for (int i = threadIdx.x; i < min(a.T * a.K, a.L) * 16; i += kFewWaves * 64) pair[i] = -1;
    find_hits(a, hits, nullptr);
    for (int p = threadIdx.x; p < a.T * a.K; p += kFewWaves * 64)
        if (le_of[p] >= 0 && first_place(a, p)) {
            const int i = index_of(hits, le_of[p]);
            pair[i * 16 + p / a.K] = (int16_t)p;
            expert[i] = (uint16_t)le_of[p];
        }
    __syncthreads();
    constexpr int kSpan = span<kFp8>::cols;
    const int64_t unit = kFp8 ? 1 : 2;
    const int l8 = lane >> 3, spans = (a.I + kSpan - 1) / kSpan, cblocks = (a.I + 127) / 128, rblocks = (a.H + 127) / 128, n_exp = n_hits(hits);
    const int units = n_exp * spans;
    const uint32_t piece = (uint32_t)(lane & 7) * 16;
    operands<kFp8, 1, 1, 2, 2> o;
    o.b[0] = array_at(a.act_hi);
    o.b[1] = array_at(a.act_lo);
#pragma unroll
    for (int i = 0; i < 2; ++i) o.row[0][i] = (uint32_t)(min(row0 + i * 8 + l8, a.H - 1) * unit * a.I) + piece;
    o.block[0] = (uint32_t)(row0 / 128 * cblocks) * 4;
    stage<kFp8, 1, 1, 2, 2> st[kFewDepth];
    bool mine[kFewDepth];
    f32x4 acc = {};
    int e = 0, s = wave, to_load = wave;     // the next span to load
    auto load = [&](int d) {
        while (s >= spans) { s -= spans; ++e; }
        const int at = min(e, n_exp - 1), le = __builtin_amdgcn_readfirstlane((int)expert[at]);
        mine[d] = pair[at * 16 + n] >= 0;
        o.w = array_at((const char *)a.down + (int64_t)le * a.H * a.I * unit);
        o.scale = array_at(kFp8 ? a.down_scale + (int64_t)le * rblocks * cblocks : nullptr);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            o.col[0][0][i] = o.col[0][1][i] = (uint32_t)(max((int)pair[at * 16 + i * 8 + l8], 0) * a.act_stride * 2) + piece;
        o.limit = to_load < units ? a.I : 0;
        st[d].load(o, s * kSpan, lane);
        s += kFewWaves;
        to_load += kFewWaves;
    };
    if (n_exp > 0) {
#pragma unroll
        for (int d = 0; d < kFewDepth - 1; ++d) load(d);
    }
    for (int u = wave; u < units; u += kFewWaves * kFewDepth) {
#pragma unroll
        for (int d = 0; d < kFewDepth; ++d) {
            load((d + kFewDepth - 1) % kFewDepth);
            if (u + d * kFewWaves < units) {
                f32x4 one[1][1] = {};
                st[d].add_to(one, lds + wave * kWaveLds<1>, lane);
                if (mine[d]) acc += one[0][0];                 // (0 times a weight that is no number is not 0)
            }
        }
    }
    float *part = (float *)lds;
    __syncthreads();
    *(f32x4 *)&part[wave * 256 + n * 16 + g * 4] = acc;
    __syncthreads();
    const int col = threadIdx.x >> 4, r = threadIdx.x & 15;
    if (col < a.T && row0 + r < a.H) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) v += part[w * 256 + threadIdx.x];
        a.out[(int64_t)col * a.out_stride + row0 + r] = mw_f32_to_bf16(v);
    }
}

// Larger batches: a pair's product by itself.  Two tiles of 16 rows share the columns' loads; two of a workgroup's four waves take
// 32 rows, every second span each.  grid: (64 rows of H, hit experts).  us of the layer with one / two / four waves to 32 rows: 256 tokens of
// 256 experts, 32 of them here, 7168 x 2048, 480 / 471 / 495; four / two: 64 tokens, four fp8 experts 46.0 / 43.9, 128 tokens of 32 experts,
// 4096 x 1024, 266 / 235.
constexpr int kDownWaves = 4, kSplit = 2;
template <bool kFp8, int kCols, int kHalves, int kDepth>
__device__ __forceinline__ void down_columns(const layer_args &a, int le, int row0, const uint16_t *list, int first, int count, char *lds)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), n = lane & 15, g = lane >> 4;
    const int64_t unit = kFp8 ? 1 : 2;
    const int cblocks = (a.I + 127) / 128, rblocks = (a.H + 127) / 128;
    const int l8 = lane >> 3;
    const uint32_t piece = (uint32_t)(lane & 7) * 16;
    operands<kFp8, 2, kCols, kHalves, 2> o;
    o.w = array_at((const char *)a.down + (int64_t)le * a.H * a.I * unit);
    o.scale = array_at(kFp8 ? a.down_scale + (int64_t)le * rblocks * cblocks : nullptr);
    o.b[0] = array_at(a.act_hi);
    o.b[1] = array_at(a.act_lo);
    o.limit = a.I;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int i = 0; i < 2; ++i) o.row[r][i] = (uint32_t)(min(row0 + r * 16 + i * 8 + l8, a.H - 1) * unit * a.I) + piece;
        o.block[r] = (uint32_t)(min(row0, a.H - 1) / 128 * cblocks) * 4;       // (32 rows from a multiple of 32)
    }
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int i = 0; i < kHalves; ++i) {
            const int at = first + c * 16 + i * 8 + l8;
            o.col[c][0][i] = o.col[c][1][i] = (uint32_t)(list[at < count ? at : first] * a.act_stride * 2) + piece;
        }
    f32x4 acc[2][kCols] = {};
    stream<kFp8, 2, kCols, kHalves, 2, kSplit, kDepth>(o, wave % kSplit, lane, lds + wave * kWaveLds<2>, acc);
    float *part = (float *)lds;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
        // part [wave][column][32 rows]
#pragma unroll
        for (int r = 0; r < 2; ++r) *(f32x4 *)&part[(wave * 16 + n) * 32 + r * 16 + g * 4] = acc[r][c];
        __syncthreads();
        constexpr int kThreads = kSplit * 64;
        for (int o = threadIdx.x % kThreads; o < 256; o += kThreads) {
            const int col = o >> 4, r = (o & 15) * 2;
            if (first + c * 16 + col >= count || row0 + r >= a.H) continue;          // (H is even)
            float v0 = 0.0f, v1 = 0.0f;
#pragma unroll
            for (int w = 0; w < kSplit; ++w) {
                const float *q = &part[((wave / kSplit * kSplit + w) * 16 + col) * 32 + r];
                v0 += q[0];
                v1 += q[1];
            }
            float *y = a.y + (int64_t)list[first + c * 16 + col] * a.H + row0 + r;
            y[0] = v0;
            y[1] = v1;
        }
        __syncthreads();
    }
}

template <bool kFp8, bool kWide>
__global__ __launch_bounds__(kDownWaves * 64) void k_layer_down(layer_args a)
{
    __shared__ __align__(16) char part[kDownWaves * kWaveLds<2>];
    __shared__ hit_set hits;
    __shared__ uint16_t list[MW_LAYER_MAX_TOKENS];
    __shared__ int n_pairs;
    find_hits(a, hits, nullptr);
    if ((int)blockIdx.y >= n_hits(hits)) return;
    const int le = nth_hit(hits, blockIdx.y), count = pairs_of(a, le, &n_pairs, list);
    const int row0 = ((int)blockIdx.x * (kDownWaves / kSplit) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) / kSplit) * 32;
    for (int first = 0; first < count;) {
        const int left = count - first;
        if (left <= 8) { down_columns<kFp8, 1, 1, kFp8 ? 3 : 4>(a, le, row0, list, first, count, part); first += 16; }
        else if (left <= 16) { down_columns<kFp8, 1, 2, kFp8 ? 2 : 3>(a, le, row0, list, first, count, part); first += 16; }
        else if (!kWide || left <= 32) { down_columns<kFp8, 2, 2, 2>(a, le, row0, list, first, count, part); first += 32; }
        else if constexpr (kWide) { down_columns<kFp8, 4, 2, 2>(a, le, row0, list, first, count, part); first += 64; }
    }
}

// out[t] = the sum of its pairs, in the order of its ids.  grid: (1024 columns, token).
__global__ __launch_bounds__(256) void k_layer_sum(layer_args a)
{
    __shared__ int use[MW_MAX_TOPK];
    const int t = blockIdx.y;
    if ((int)threadIdx.x < a.K) le_of[threadIdx.x] = (int16_t)local_slot(a, a.eslot, a.ids[t * a.K + threadIdx.x]);
    __syncthreads();
    if ((int)threadIdx.x < a.K) use[threadIdx.x] = le_of[threadIdx.x] >= 0 && first_place(a, threadIdx.x);
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
int64_t act_stride(int64_t inter) { return mw_align_up(inter, 64) + 128; }
layer_ws layer_layout(const mw_ctx *ctx, int64_t inter, int64_t tokens)
{
    layer_ws w;
    int64_t o = 0;
    const int64_t pairs = tokens * ctx->cfg.top_k;
    w.hi = o; o += mw_align_up(2 * pairs * act_stride(inter), 256);
    w.lo = o; o += mw_align_up(2 * pairs * act_stride(inter), 256);
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
    if (!fp8 && (e->gate_up_scale_dev || e->down_scale_dev)) return MW_ERR_INVALID_ARG;
    if (fp8 && ctx->n_local > 0 && (!e->gate_up_scale_dev || !e->down_scale_dev)) return MW_ERR_INVALID_ARG;      // (a rank without experts has no arrays)
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
    // places inside an expert's matrices, the tokens and their activations are 32-bit, below 2^31
    const int64_t far = 2LL << 30, tokens = n_tokens, unit = experts->format == MW_ROW_FP8_E4M3_BLOCK128 ? 1 : 2;
    if (2 * unit * H * I > far || (tokens > 0 && x_stride > far / 2 / tokens) || 2 * act_stride(I) * tokens * ctx->cfg.top_k > far) return MW_ERR_UNSUPPORTED;
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
    a.act_stride = act_stride(I);
    a.act_hi = (uint16_t *)(b + w.hi); a.act_lo = (uint16_t *)(b + w.lo); a.y = (float *)(b + w.y);
    a.out = (uint16_t *)out_dev; a.out_stride = out_stride;
    a.flags = error_flags_dev;
    const hipStream_t s = (hipStream_t)stream;
    const int64_t pairs = (int64_t)n_tokens * a.K;
    const uint32_t hits = (uint32_t)(a.L < 1 ? 1 : pairs < a.L ? pairs : a.L);       // experts that can be hit at most
    const uint32_t ids_lds = (uint32_t)mw_align_up(2 * pairs, 16);
    const dim3 up((uint32_t)((I + 15) / 16), hits);
    const bool fp8 = experts->format == MW_ROW_FP8_E4M3_BLOCK128;
    // An expert's weights are read once for up to 32 of its tokens, or (bf16) for up to 64 at half the waves a CU holds, where experts have
    // 24 tokens on average.  us, 32 / 64: 256 tokens, 8 experts, top-2, 4096 x 2048 227 / 177; 16 experts, top-2 258 / 209; 16 experts, top-4,
    // 4096 x 1024 239 / 184.  fp8 would need 272 and 423 registers for 64: the same three 166 / 169, 184 / 207, 177 / 192; 128 tokens, 32 experts,
    // top-8, 213 / 277.
    const bool wide = !fp8 && pairs >= 24LL * a.E;
    if (fp8) hipLaunchKernelGGL((k_layer_up<true, false>), up, dim3(kUpWaves * 64), ids_lds, s, a);
    else if (wide) hipLaunchKernelGGL((k_layer_up<false, true>), up, dim3(kUpWaves * 64), ids_lds, s, a);
    else hipLaunchKernelGGL((k_layer_up<false, false>), up, dim3(kUpWaves * 64), ids_lds, s, a);
    MW_HIP_CHECK(hipGetLastError());
    // Up to 16 tokens the second product adds an output up over its experts; beyond it, or for any batch: pairs, then k_layer_sum.  us, this way / that
    // way, bf16: 1 token, 64 experts, top-8, 4096 x 1024 45.2 / 49.5; 4 tokens, 16 experts, top-2 40.7 / 43.3; 16 tokens, top-4 74.7 / 77.1.  By tokens
    // alone it is a coarse rule: over 60 sizes of 1 to 16 tokens it wins up to 20 % (1 token, top-6 of 128, 2048 x 768 18.7 / 22.6) where few experts
    // are hit, and loses where many are or in fp8: 16 tokens, top-8 of 64, 2048 x 512 88.8 / 82.8, in fp8 71.6 / 69.7; 32 fp8 experts of 256 here, 7168 x
    // 2048, 16 tokens 118 / 104, 2 tokens 34.5 / 30.6.
    if (n_tokens <= 16) {
        const dim3 down((uint32_t)((H + 15) / 16));
        const uint32_t lds = ids_lds + hits * 34;
        if (fp8) hipLaunchKernelGGL((k_layer_down_few<true>), down, dim3(kFewWaves * 64), lds, s, a);
        else hipLaunchKernelGGL((k_layer_down_few<false>), down, dim3(kFewWaves * 64), lds, s, a);
        MW_HIP_CHECK(hipGetLastError());
        return MW_OK;
    }
    const dim3 down((uint32_t)((H + 63) / 64), hits);
    if (fp8) hipLaunchKernelGGL((k_layer_down<true, false>), down, dim3(kDownWaves * 64), ids_lds, s, a);
    else if (wide) hipLaunchKernelGGL((k_layer_down<false, true>), down, dim3(kDownWaves * 64), ids_lds, s, a);
    else hipLaunchKernelGGL((k_layer_down<false, false>), down, dim3(kDownWaves * 64), ids_lds, s, a);
    MW_HIP_CHECK(hipGetLastError());
    hipLaunchKernelGGL(k_layer_sum, dim3((uint32_t)((H + 1023) / 1024), (uint32_t)n_tokens), dim3(256), 2 * MW_MAX_TOPK, s, a);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
