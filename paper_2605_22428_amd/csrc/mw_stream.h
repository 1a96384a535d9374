// Products of matrix rows that are streamed from memory with a few columns (tokens): the layer's experts, the adapters' first factors.
#ifndef MW_STREAM_H_
#define MW_STREAM_H_

#include "mw_math.h"

namespace {

// A wave takes 128 bytes of each of 16 weight rows at a time (64 bf16 or 128 fp8 columns) with two loads, eight whole cache lines
// each, and the tokens' columns that belong to them likewise; they pass through a piece of LDS of the wave's own, out of which come the matrix
// instruction's operands.  Loaded straight into operand layout, 16 rows by 64 bytes a load, the weights of 1.9 GB came at 6.3 TB/s with nothing
// else to load, and tokens loaded so beside them cost as much again a load (up 5.0, down 3.25 TB/s); whole lines, streaming, come at 7.0 TB/s.
constexpr int kPitch = 144;              // bytes from row to row in LDS: 16 rows start on different banks
constexpr int kTileBytes = 16 * kPitch;
template <bool kFp8> struct span { static constexpr int cols = kFp8 ? 128 : 64, pieces = kFp8 ? 2 : 1; };     // pieces of 64 columns

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// Eight e4m3 codes as bf16 (every e4m3 value is a bf16 value).
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b)
{
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    bf16x8 r;
    r[0] = p0[0]; r[1] = p0[1]; r[2] = p1[0]; r[3] = p1[1]; r[4] = p2[0]; r[5] = p2[1]; r[6] = p3[0]; r[7] = p3[1];
    return r;
}
// LDS written by lanes of this wave is read by others of it: the accesses stay in program order (the hardware keeps them so).
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// An array whose loads past its end are zeros and cost no traffic: places are 32-bit, and kNowhere plus any place (below 2^31) is past it.
// So every load of the stream is issued whether there is something to load or not; a load behind a branch would make each wait
// behind the branch wait for it (the counter of loads on the way has to suit both ways), and with that for all of them.
typedef __amdgpu_buffer_rsrc_t array;
constexpr uint32_t kNowhere = 0x80000000u;
__device__ __forceinline__ array array_at(const void *p) { return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)kNowhere, 0x00027000); }
template <bool kStreaming>
__device__ __forceinline__ u32x4 load16(array from, uint32_t at)
{
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, kStreaming ? 2 : 0));
}

// Rows and columns of a product.  A lane's places: of row lane / 8 and 8 + lane / 8 of every tile, at byte (lane % 8) * 16.
template <bool kFp8, int kRows, int kCols, int kHalves, int kTerms>
struct operands {
    array w, scale, b[kTerms];
    uint32_t row[kRows][2], col[kCols][kTerms][kHalves], block[kRows];      // block: byte of the rows' first scale
    int limit;                                                              // columns
};

// kHalves 1: no tile has more than eight tokens, the second load of theirs is left out.  kOnce: what is read once, the rows or the columns
// (the other is left to the caches).
enum { kOnceRows, kOnceCols };
template <bool kFp8, int kRows, int kCols, int kHalves, int kTerms, int kOnce = kOnceRows>
struct stage {
    static constexpr int kPieces = span<kFp8>::pieces;
    u32x4 w[kRows][2];
    u32x4 b[kCols][kTerms][kPieces][kHalves];
    uint32_t s[kRows];
    __device__ __forceinline__ void load(const operands<kFp8, kRows, kCols, kHalves, kTerms> &o, int k0, int lane)
    {
        const uint32_t at = (uint32_t)(lane & 7) * 16, end = kFp8 ? (uint32_t)o.limit : 2u * (uint32_t)o.limit;
        const uint32_t byte = kFp8 ? (uint32_t)k0 : 2u * (uint32_t)k0, w_at = byte + at < end ? byte : kNowhere;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
#pragma unroll
            for (int i = 0; i < 2; ++i) w[r][i] = load16<kOnce == kOnceRows>(o.w, o.row[r][i] + w_at);
            if constexpr (kFp8) s[r] = __builtin_amdgcn_raw_buffer_load_b32(o.scale, k0 < o.limit ? o.block[r] + (uint32_t)(k0 >> 7) * 4 : kNowhere, 0, 0);
        }
#pragma unroll
        for (int h = 0; h < kPieces; ++h) {
            const uint32_t b_byte = 2u * (uint32_t)k0 + (uint32_t)h * 128, b_at = b_byte + at < 2u * (uint32_t)o.limit ? b_byte : kNowhere;
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
                for (int t = 0; t < kTerms; ++t)
#pragma unroll
                    for (int i = 0; i < kHalves; ++i) b[c][t][h][i] = load16<kOnce == kOnceCols>(o.b[t], o.col[c][t][i] + b_at);
        }
    }
    __device__ __forceinline__ void add_to(f32x4 (&acc)[kRows][kCols], char *lds, int lane) const
    {
        char *to = lds + (lane >> 3) * kPitch + (lane & 7) * 16;
        const char *from = lds + (lane & 15) * kPitch + (lane >> 4) * 16;
        bf16x8 v[kRows][2 * kPieces];
        wave_order();
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i) *(u32x4 *)(to + r * kTileBytes + i * 8 * kPitch) = w[r][i];
        wave_order();
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const u32x4 q = *(const u32x4 *)(from + r * kTileBytes + j * 64);
                // bf16: columns j * 32 + g * 8 ..; fp8: columns j * 64 + g * 16 .., eight for each of two instructions
                if constexpr (kFp8) { v[r][j * 2] = widen(q.x, q.y); v[r][j * 2 + 1] = widen(q.z, q.w); }
                else v[r][j] = __builtin_bit_cast(bf16x8, q);
            }
        f32x4 part[kRows][kCols];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int c = 0; c < kCols; ++c) part[r][c] = kFp8 ? f32x4{} : acc[r][c];
#pragma unroll
        for (int h = 0; h < kPieces; ++h)
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
                for (int t = 0; t < kTerms; ++t) {
                    char *tile = lds + kRows * kTileBytes;
                    wave_order();
#pragma unroll
                    for (int i = 0; i < kHalves; ++i) *(u32x4 *)(tile + (to - lds) + i * 8 * kPitch) = b[c][t][h][i];
                    wave_order();
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const char *x = tile + (lane & 15) * kPitch + (kFp8 ? (lane >> 4) * 32 + j * 16 : (lane >> 4) * 16 + j * 64);
                        const bf16x8 xv = *(const bf16x8 *)x;
#pragma unroll
                        for (int r = 0; r < kRows; ++r) part[r][c] = mma(v[r][h * 2 + j], xv, part[r][c]);
                    }
                }
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                if constexpr (kFp8) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[r][c][i] += __uint_as_float(s[r]) * part[r][c][i];
                } else {
                    acc[r][c] = part[r][c];
                }
            }
    }
};
template <int kRows> constexpr int kWaveLds = (kRows + 1) * kTileBytes;

// acc += rows times columns; the workgroup's waves take every kWaves-th span each, kDepth of them on the way at a time.
template <bool kFp8, int kRows, int kCols, int kHalves, int kTerms, int kWaves, int kDepth, int kOnce = kOnceRows>
__device__ __forceinline__ void stream(const operands<kFp8, kRows, kCols, kHalves, kTerms> &o, int wave, int lane, char *lds, f32x4 (&acc)[kRows][kCols])
{
    constexpr int kSpan = span<kFp8>::cols;
    stage<kFp8, kRows, kCols, kHalves, kTerms, kOnce> st[kDepth];
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) st[d].load(o, (wave + d * kWaves) * kSpan, lane);
    for (int k0 = wave * kSpan; k0 < o.limit; k0 += kWaves * kDepth * kSpan) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            st[(d + kDepth - 1) % kDepth].load(o, k0 + (d + kDepth - 1) * kWaves * kSpan, lane);
            if (k0 + d * kWaves * kSpan < o.limit) st[d].add_to(acc, lds, lane);
        }
    }
}

}  // namespace

#endif  // MW_STREAM_H_
