// mw_route, mw_route_backward: a token's gate scores -> the K experts it goes to and their weights, and the way back.
//
// One wave a token, its scores in registers (lane l holds experts l, l + 64, ...).  The K best are taken one by one: a wave-wide
// maximum of keys that order like the scores, the lowest expert among equals.  By score and bias nothing but one float addition decides which
// experts are taken, so the ids are the same whatever the order of the sums in the weights; by share a sigmoid or an exponential and a sum
// decide as well, in fp32, and experts closer than their rounding may change places.  Measured on one MI355X: 8192 tokens, 256 experts in 8
// groups, top-8 (8.9 MB) 10.5 us: eight rounds of a wave's maximum are some 700 instructions a token, which bound it, not the bytes
// (1.3 us of them); by share 11.6, of a softmax gate 12.7 (by score 11.1); backward of 4096 tokens (4.5 MB) 6.4 us, 5 of them the kernel.  Smaller calls are a launch, 5 to 6 us in a stream of them.
#include <float.h>

#include "mw_math.h"

namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;

struct gate_args {
    const void *logits;
    int64_t stride;             // elements from one token's scores to the next's
    const float *bias;
    int32_t n_tokens, n_experts, top_k, score, by_share, n_groups, kept, group_size;
    int32_t group_lanes;        // lanes that look at a group together
    uint32_t group_mul;         // expert / group_size = expert * group_mul >> 20 (experts below 1024)
    float scale;
};

template <bool kBf16>
__device__ __forceinline__ float load_score(const void *p, int64_t at)
{
    // NaN counts as -inf, +inf as the largest finite value
    const float v = kBf16 ? mw_bf16_to_f32(((const uint16_t *)p)[at]) : ((const float *)p)[at];
    return v != v ? -INFINITY : fminf(v, FLT_MAX);
}

// The largest of the lanes' scores, no lower than the lowest finite value; every lane active.
__device__ __forceinline__ float wave_top(float l) { return mw_key_value(mw_wave_max(mw_order_key(fmaxf(l, -FLT_MAX)))); }

// What the experts taken weigh in a sigmoid gate, up to a factor: lane k the k-th, 0 where there is none.  That is sig(l), or, where one is below -87,
// sig(l) / exp(min(top, 0)) with the largest score: from there down sig has lost bits in 32 bits, and from -104 down it is 0, where shares of a token
// whose scores are all that low still are ordinary numbers.  Below -708 sig is under the smallest normal number of 64 bits and counts as 0: such
// scores stand for masks (-1e4, a type's lowest value).  8192 tokens, top-8: 10.5 us, always divided 10.8.
__device__ __forceinline__ float sigmoids(float l, bool taken)
{
    float v = taken ? 1.0f / (1.0f + expf(-l)) : 0.0f;
    if (__ballot(taken && l < -87.0f)) {
        const float top = wave_top(l);
        v = taken && l >= -708.0f ? expf(fminf(l, 0.0f) - fminf(top, 0.0f)) / (1.0f + expf(-fabsf(l))) : 0.0f;
    }
    return v;
}

// What selection goes by, before the bias, where the gate takes experts by their shares: sigmoids, or the softmax over all experts.  An expert
// that cannot be taken keeps -inf.
template <int kVals>
__device__ __forceinline__ void shares(const gate_args &a, const float (&l)[kVals], float (&share)[kVals])
{
    if (a.score == MW_GATE_SIGMOID_TOPK) {
#pragma unroll
        for (int j = 0; j < kVals; ++j) share[j] = l[j] > -INFINITY ? 1.0f / (1.0f + expf(-l[j])) : -INFINITY;
        return;
    }
    float m = l[0], sum = 0.0f;
#pragma unroll
    for (int j = 1; j < kVals; ++j) m = fmaxf(m, l[j]);
    m = wave_top(m);
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
        share[j] = expf(l[j] - m);
        sum += share[j];
    }
    const float total = mw_wave_sum_f32(sum);
#pragma unroll
    for (int j = 0; j < kVals; ++j) share[j] = l[j] > -INFINITY ? share[j] / total : -INFINITY;
}

// Keys of the scores that selection goes by, 0 where an expert cannot be taken.
template <int kVals>
__device__ __forceinline__ void select_keys(const gate_args &a, const float (&l)[kVals], uint32_t (&key)[kVals], int lane, float *row)
{
    float s[kVals], by[kVals];
#pragma unroll
    for (int j = 0; j < kVals; ++j) by[j] = l[j];
    if (a.by_share) shares<kVals>(a, l, by);
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
        const int e = j * 64 + lane;
        s[j] = -INFINITY;
        if (e < a.n_experts) {
            s[j] = a.bias ? by[j] + a.bias[e] : by[j];
            s[j] = s[j] != s[j] ? -INFINITY : fminf(s[j], FLT_MAX) + 0.0f;      // (+ 0: -0 and 0 are one value)
        }
        key[j] = s[j] > -INFINITY ? mw_order_key(s[j]) : 0u;
    }
    if (a.n_groups == 1) return;
    // Several lanes a group, a power of two: its two best scores, then how many groups are ahead of it.
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
        const int e = j * 64 + lane;
        if (e < a.n_experts) row[e] = s[j];
    }
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    float best = -INFINITY, second = -INFINITY;
    const int G = a.n_groups, S = a.group_size, P = a.group_lanes, group = lane / P;
    if (group < G) {
#pragma unroll 4
        for (int i = lane % P; i < S; i += P) {
            const float v = row[group * S + i];
            second = fmaxf(second, fminf(best, v));
            best = fmaxf(best, v);
        }
    }
    for (int d = 1; d < P; d *= 2) {
        const float ob = __shfl_xor(best, d), os = __shfl_xor(second, d);
        second = fmaxf(fmaxf(second, os), fminf(best, ob));
        best = fmaxf(best, ob);
    }
    // A group's rank as a key; 0, behind every score, for one none of whose experts can be taken (a score can be -inf with one that can).
    // By shares the scores of the experts that can be taken count: two of a sigmoid gate, one of a softmax gate.
    const bool one = a.by_share ? a.score != MW_GATE_SIGMOID_TOPK || !(second > -INFINITY) : S == 1;
    const uint32_t rank = best > -INFINITY ? mw_order_key(one ? best : best + second) : 0u;
    const uint32_t mine = (uint32_t)__shfl((int)rank, min(lane * P, 63));      // lane g: group g
    int ahead = 0;
    for (int g = 0; g < G; ++g) {
        const uint32_t other = (uint32_t)__builtin_amdgcn_readlane((int)mine, g);
        ahead += other > mine || (other == mine && g < lane) ? 1 : 0;
    }
    const unsigned long long kept = __ballot(lane < G && ahead < a.kept);
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
        const uint32_t g = ((uint32_t)(j * 64 + lane) * a.group_mul) >> 20;
        if (!((kept >> (g & 63u)) & 1ull)) key[j] = 0u;
    }
}

template <int kVals, bool kBf16>
__global__ __launch_bounds__(kBlock) void k_route(gate_args a, int32_t *__restrict__ ids, float *__restrict__ weights)
{
    __shared__ float rows[kWaves][kVals * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t t = (int64_t)blockIdx.x * kWaves + wave;
    if (t >= a.n_tokens) return;
    float l[kVals];
    uint32_t key[kVals];
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
        const int e = j * 64 + lane;
        l[j] = e < a.n_experts ? load_score<kBf16>(a.logits, t * a.stride + e) : -INFINITY;
    }
    select_keys<kVals>(a, l, key, lane, rows[wave]);

    int my_id = -1;                              // lane k: the k-th choice
    for (int k = 0; k < a.top_k; ++k) {
        uint32_t best = key[0];
        int at = 0;
#pragma unroll
        for (int j = 1; j < kVals; ++j)
            if (key[j] > best) { best = key[j]; at = j; }
        const uint32_t top = mw_wave_max(best);
        if (top == 0u) break;
        const unsigned long long equal = __ballot(best == top);
        int owner = __builtin_ctzll(equal);
        if (equal & (equal - 1)) {               // several lanes hold it: the lowest expert
            const uint32_t low = mw_wave_max(best == top ? 0xffffu - (uint32_t)(at * 64 + lane) : 0u);
            owner = (int)((0xffffu - low) & 63u);
        }
        const int id = __builtin_amdgcn_readlane(at, owner) * 64 + owner;
        if (lane == k) my_id = id;
        const int gone = lane == owner ? at : -1;
#pragma unroll
        for (int j = 0; j < kVals; ++j) key[j] = j == gone ? 0u : key[j];
    }
    // The choices' scores, by way of LDS: carried through the rounds they would be three instructions of each.
    float *row = rows[wave];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < kVals; ++j) row[j * 64 + lane] = l[j];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    __builtin_amdgcn_wave_barrier();
    const float my_l = my_id >= 0 ? row[my_id] : -INFINITY;

    float v, total;
    if (a.score == MW_GATE_SIGMOID_TOPK) {
        v = sigmoids(my_l, my_id >= 0);
        total = mw_wave_sum_f32(v);
    } else {
        float m = my_id >= 0 ? my_l : -INFINITY;
        if (a.score == MW_GATE_SOFTMAX) {
#pragma unroll
            for (int j = 0; j < kVals; ++j) m = fmaxf(m, l[j]);
        }
        m = wave_top(m);
        v = my_id >= 0 ? expf(my_l - m) : 0.0f;
        float sum = v;
        if (a.score == MW_GATE_SOFTMAX) {
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < kVals; ++j) sum += expf(l[j] - m);
        }
        total = mw_wave_sum_f32(sum);
    }
    if (lane < a.top_k) {
        ids[t * a.top_k + lane] = my_id;
        weights[t * a.top_k + lane] = total > 0.0f ? v / total * a.scale : 0.0f;
    }
}

template <int kVals, bool kBf16>
__global__ __launch_bounds__(kBlock) void k_route_backward(gate_args a, const int32_t *__restrict__ ids, const float *__restrict__ d_weights,
                                                           void *__restrict__ d_logits, int64_t d_stride)
{
    __shared__ float rows[kWaves][kVals * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t t = (int64_t)blockIdx.x * kWaves + wave;
    if (t >= a.n_tokens) return;
    float *row = rows[wave];
    int id = -1;
    float g = 0.0f;
    if (lane < a.top_k) {
        id = ids[t * a.top_k + lane];
        if (id < 0 || id >= a.n_experts) id = -1;
        else g = d_weights[t * a.top_k + lane];
    }
    const float my_l = id >= 0 ? load_score<kBf16>(a.logits, t * a.stride + id) : -INFINITY;
    float l[kVals];
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
        const int e = j * 64 + lane;
        l[j] = -INFINITY;
        if (a.score == MW_GATE_SOFTMAX && e < a.n_experts) l[j] = load_score<kBf16>(a.logits, t * a.stride + e);
        if (e < kVals * 64) row[e] = 0.0f;
    }
    // q: the weight before the factor; `add` goes to the expert's place
    float q, add, inv = 0.0f, m = 0.0f;
    if (a.score == MW_GATE_SIGMOID_TOPK) {
        const float v = sigmoids(my_l, id >= 0);
        const float total = mw_wave_sum_f32(v);
        q = total > 0.0f ? v / total : 0.0f;
        add = q * (1.0f / (1.0f + expf(my_l)));             // (1 - sigmoid, with small ones kept)
        if (id < 0) add = 0.0f;
    } else {
        m = my_l;
#pragma unroll
        for (int j = 0; j < kVals; ++j) m = fmaxf(m, l[j]);
        m = wave_top(m);
        const float v = id >= 0 ? expf(my_l - m) : 0.0f;
        float sum = v;
        if (a.score == MW_GATE_SOFTMAX) {
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < kVals; ++j) sum += expf(l[j] - m);
        }
        const float total = mw_wave_sum_f32(sum);
        inv = total > 0.0f ? 1.0f / total : 0.0f;
        q = v * inv;
        add = q;
    }
    const float mean = mw_wave_sum_f32(g * q);
    if (a.score == MW_GATE_SOFTMAX) add = g;                // gradients by expert; the rest below
    else add *= a.scale * (g - mean);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    __builtin_amdgcn_wave_barrier();
    if (id >= 0) atomicAdd(&row[id], add);                  // (an expert named twice: both)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
        const int e = j * 64 + lane;
        if (e >= a.n_experts) continue;
        float d = row[e];
        if (a.score == MW_GATE_SOFTMAX) d = a.scale * (expf(l[j] - m) * inv) * (d - mean);
        if constexpr (kBf16) ((uint16_t *)d_logits)[t * d_stride + e] = mw_f32_to_bf16(d);
        else ((float *)d_logits)[t * d_stride + e] = d;
    }
}

int32_t gate_ready(const mw_ctx *ctx, const mw_gate *gate, const void *logits, int32_t format, int64_t stride, int32_t n_tokens, gate_args *a)
{
    if (!gate || n_tokens < 0 || ctx->cfg.n_experts < 1) return MW_ERR_INVALID_ARG;
    const int32_t E = ctx->cfg.n_experts;
    if (E > MW_GATE_MAX_EXPERTS) return MW_ERR_UNSUPPORTED;
    if (n_tokens > ctx->cfg.max_tokens) return MW_ERR_CAPACITY;
    const int32_t score = gate->score & ~MW_GATE_BY_SHARE;
    if (score < MW_GATE_SOFTMAX || score > MW_GATE_SIGMOID_TOPK) return MW_ERR_INVALID_ARG;
    if (format != MW_LOGITS_F32 && format != MW_LOGITS_BF16) return MW_ERR_INVALID_ARG;
    if (gate->n_groups < 1 || gate->kept_groups < 1 || gate->kept_groups > gate->n_groups || E % gate->n_groups != 0) return MW_ERR_INVALID_ARG;
    if (gate->n_groups > MW_GATE_MAX_GROUPS) return MW_ERR_UNSUPPORTED;
    if (!(gate->scale - gate->scale == 0.0f)) return MW_ERR_INVALID_ARG;          // (a finite factor)
    if (stride < E) return MW_ERR_INVALID_ARG;
    const uintptr_t unit = format == MW_LOGITS_F32 ? 3u : 1u;
    if (n_tokens > 0 && (!logits || ((uintptr_t)logits & unit))) return MW_ERR_INVALID_ARG;
    a->logits = logits; a->stride = stride; a->bias = nullptr;
    a->n_tokens = n_tokens; a->n_experts = E; a->top_k = ctx->cfg.top_k;
    a->score = score; a->by_share = gate->score != score; a->n_groups = gate->n_groups; a->kept = gate->kept_groups; a->scale = gate->scale;
    a->group_size = E / gate->n_groups;
    a->group_lanes = 1;
    while (a->group_lanes * 2 * gate->n_groups <= 64 && a->group_lanes * 2 <= a->group_size) a->group_lanes *= 2;
    a->group_mul = ((1u << 20) + (uint32_t)a->group_size - 1) / (uint32_t)a->group_size;
    return MW_OK;
}

// The instance for the context's experts: values a lane, 1 to 16.
#define MW_GATE_LAUNCH(kernel, bf16, grid, s, ...)                                                                   \
    do {                                                                                                             \
        const int vals_ = (a.n_experts + 63) / 64;                                                                   \
        if (vals_ <= 1) hipLaunchKernelGGL((kernel<1, bf16>), grid, dim3(kBlock), 0, s, __VA_ARGS__);                \
        else if (vals_ <= 2) hipLaunchKernelGGL((kernel<2, bf16>), grid, dim3(kBlock), 0, s, __VA_ARGS__);           \
        else if (vals_ <= 4) hipLaunchKernelGGL((kernel<4, bf16>), grid, dim3(kBlock), 0, s, __VA_ARGS__);           \
        else if (vals_ <= 8) hipLaunchKernelGGL((kernel<8, bf16>), grid, dim3(kBlock), 0, s, __VA_ARGS__);           \
        else hipLaunchKernelGGL((kernel<16, bf16>), grid, dim3(kBlock), 0, s, __VA_ARGS__);                          \
    } while (0)

}  // namespace

extern "C" MW_API int32_t mw_route(mw_ctx *ctx, const mw_gate *gate, const void *logits_dev, int32_t logit_format, int64_t logit_stride,
                                   const float *bias_dev, int32_t n_tokens, int32_t *topk_ids_dev, float *topk_weights_dev, void *stream)
{
    if (!ctx) return MW_ERR_INVALID_ARG;
    gate_args a;
    int32_t rc = gate_ready(ctx, gate, logits_dev, logit_format, logit_stride, n_tokens, &a);
    if (rc == MW_OK) rc = mw_on_device_of(ctx);
    if (rc != MW_OK) return rc;
    if (n_tokens == 0) return MW_OK;
    if (!topk_ids_dev || !topk_weights_dev) return MW_ERR_INVALID_ARG;
    a.bias = bias_dev;
    const dim3 grid((uint32_t)((n_tokens + kWaves - 1) / kWaves));
    if (logit_format == MW_LOGITS_BF16) MW_GATE_LAUNCH(k_route, true, grid, (hipStream_t)stream, a, topk_ids_dev, topk_weights_dev);
    else MW_GATE_LAUNCH(k_route, false, grid, (hipStream_t)stream, a, topk_ids_dev, topk_weights_dev);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}

extern "C" MW_API int32_t mw_route_backward(mw_ctx *ctx, const mw_gate *gate, const void *logits_dev, int32_t logit_format, int64_t logit_stride,
                                            const int32_t *topk_ids_dev, const float *d_weights_dev, int32_t n_tokens, void *d_logits_dev,
                                            int64_t d_logit_stride, void *stream)
{
    if (!ctx) return MW_ERR_INVALID_ARG;
    gate_args a;
    int32_t rc = gate_ready(ctx, gate, logits_dev, logit_format, logit_stride, n_tokens, &a);
    if (rc == MW_OK) rc = mw_on_device_of(ctx);
    if (rc != MW_OK) return rc;
    if (d_logit_stride < a.n_experts) return MW_ERR_INVALID_ARG;
    if (n_tokens == 0) return MW_OK;
    if (!topk_ids_dev || !d_weights_dev || !d_logits_dev) return MW_ERR_INVALID_ARG;
    if ((uintptr_t)d_logits_dev & (logit_format == MW_LOGITS_F32 ? 3u : 1u)) return MW_ERR_INVALID_ARG;
    const dim3 grid((uint32_t)((n_tokens + kWaves - 1) / kWaves));
    const hipStream_t s = (hipStream_t)stream;
    if (logit_format == MW_LOGITS_BF16) MW_GATE_LAUNCH(k_route_backward, true, grid, s, a, topk_ids_dev, d_weights_dev, d_logits_dev, d_logit_stride);
    else MW_GATE_LAUNCH(k_route_backward, false, grid, s, a, topk_ids_dev, d_weights_dev, d_logits_dev, d_logit_stride);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}
