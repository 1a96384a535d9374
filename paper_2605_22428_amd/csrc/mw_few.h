// Products of matrices with a few rows each: the matrices' bytes bound them, every matrix row is read once and used for sixteen rows at a time.
#ifndef MW_FEW_H_
#define MW_FEW_H_

#include "mw_stream.h"
#include "mw_tile.h"

namespace {

// Sixteen matrix rows are one side of the matrix instruction, up to sixteen rows the other.  Waves that share a tile take every kAlong-th 128 bytes along the sum, kDepth of
// them on the way at a time, as mw_stream.h does and for its reasons; bf16 values and codes differ in the instruction only.
template <bool kInt8> struct few_kind;
template <> struct few_kind<false> {
    typedef f32x4 acc;
    static __device__ __forceinline__ acc mma(u32x4 a, u32x4 b, acc c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0); }
};
template <> struct few_kind<true> {
    typedef i32x4 acc;
    static __device__ __forceinline__ acc mma(u32x4 a, u32x4 b, acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0); }
};
constexpr int kSpanBytes = 128;
// Weights from memory, a call with all its launches: 32 rows of four experts 7168 x 2048, 352 MB, 63 us (5.6 TB/s); 64 of eight 4096 x 1024, 201 MB, 42 us (4.8); their codes, 101 MB, 28 us with
// both quantisations.  One row of one expert 4096 x 1024, 25 MB: 7.2 and 4.6 us, which are launches and three dependent round trips (offsets, weights, results).

template <int kCols> struct few_operands {
    array w, x;
    uint32_t row[2], col[kCols][2], limit;       // bytes; a lane's rows are lane / 8 and 8 + lane / 8, its piece byte (lane % 8) * 16
};
template <bool kInt8, int kCols>
struct few_stage {
    u32x4 w[2], x[kCols][2];
    __device__ __forceinline__ void load(const few_operands<kCols> &o, uint32_t byte, int lane)
    {
        const bool in = byte + (uint32_t)(lane & 7) * 16 < o.limit;
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = load16<true>(o.w, in && o.row[i] != kNowhere ? o.row[i] + byte : kNowhere);
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) x[c][i] = load16<false>(o.x, in && o.col[c][i] != kNowhere ? o.col[c][i] + byte : kNowhere);
    }
    __device__ __forceinline__ void add_to(typename few_kind<kInt8>::acc (&acc)[kCols], char *lds, int lane) const
    {
        char *to = lds + (lane >> 3) * kPitch + (lane & 7) * 16;
        const char *from = lds + (lane & 15) * kPitch + (lane >> 4) * 16;
        u32x4 v[2];
        wave_order();
#pragma unroll
        for (int i = 0; i < 2; ++i) *(u32x4 *)(to + i * 8 * kPitch) = w[i];
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) *(u32x4 *)(to + (c + 1) * kTileBytes + i * 8 * kPitch) = x[c][i];
        wave_order();
#pragma unroll
        for (int j = 0; j < 2; ++j) v[j] = *(const u32x4 *)(from + j * 64);
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[c] = few_kind<kInt8>::mma(v[j], *(const u32x4 *)(from + (c + 1) * kTileBytes + j * 64), acc[c]);
    }
};

// Sixteen matrix rows of tile `tile` times rows first .. of run e (count of them left).  Op::kTerms 2: rows are sums of two, the second K values behind the first; both are
// columns of the matrix instruction, which has sixteen whether they are used or not.
template <class Op, int kAlong, int kCols, int kDepth>
__device__ __forceinline__ void few_columns(const typename Op::args &a, int e, int tile, int64_t first, int count, char *lds)
{
    typedef few_kind<Op::kInt8> kind;
    const int lane = threadIdx.x & 63, wave = kAlong > 1 ? __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) : 0, l8 = lane >> 3;
    const uint32_t piece = (uint32_t)(lane & 7) * 16;
    constexpr int kUnit = Op::kInt8 ? 1 : 2, kTerms = Op::kTerms, kPass = kCols * 16 / kTerms;
    few_operands<kCols> o;
    o.w = array_at(Op::few_matrix(a, e, tile));          // (of the tile on: a matrix may be larger than an array's 2 GiB)
    o.x = array_at(Op::few_x(a, first));
    o.limit = (uint32_t)a.K * kUnit;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t at = Op::few_row(a, tile, i * 8 + l8);
        o.row[i] = at == kNowhere ? at : at + piece;
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            const int column = c * 16 + i * 8 + l8, r = column % kPass, term = column / kPass;
            o.col[c][i] = r < count ? ((uint32_t)r * (uint32_t)a.x_stride + (uint32_t)(term * a.K)) * kUnit + piece : kNowhere;
        }
    }
    typename kind::acc acc[kCols] = {};
    few_stage<Op::kInt8, kCols> st[kDepth];
    char *mine = lds + wave * (kCols + 1) * kTileBytes;
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) st[d].load(o, (uint32_t)(wave + d * kAlong) * kSpanBytes, lane);
    for (uint32_t byte = (uint32_t)wave * kSpanBytes; byte < o.limit; byte += kAlong * kDepth * kSpanBytes) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            st[(d + kDepth - 1) % kDepth].load(o, byte + (uint32_t)(d + kDepth - 1) * kAlong * kSpanBytes, lane);
            if (byte + (uint32_t)d * kAlong * kSpanBytes < o.limit) st[d].add_to(acc, mine, lane);
        }
    }
    typedef decltype(acc[0][0] + acc[0][0]) value;
    value *part = (value *)lds;                  // [wave][column][16 rows]
    if constexpr (kTerms == 2 && kCols == 2) acc[0] += acc[1];
    auto order = [] { if constexpr (kAlong > 1) __syncthreads(); else wave_order(); };
    constexpr int kSums = kTerms == 2 ? 1 : kCols, kHere = kPass < 16 ? kPass : 16;
#pragma unroll
    for (int c = 0; c < kSums; ++c) {
        order();                                 // (the sums take the place of the waves' pieces)
        *(typename kind::acc *)&part[(wave * 16 + (lane & 15)) * 16 + (lane >> 4) * 4] = acc[c];
        order();
        constexpr int kEach = Op::kPair ? 8 : 16;
        for (int t = (int)threadIdx.x % (64 * kAlong); t < kHere * kEach; t += 64 * kAlong) {
            const int col = t / kEach, r = t % kEach;
            if (c * 16 + col >= count) continue;
            value v = 0, w = 0;
#pragma unroll
            for (int n = 0; n < kAlong; ++n) {
                v += part[(n * 16 + col) * 16 + r];
                if constexpr (kTerms == 2 && kCols == 1) v += part[(n * 16 + 8 + col) * 16 + r];
                if constexpr (Op::kPair) w += part[(n * 16 + col) * 16 + 8 + r];
            }
            Op::few_emit(a, e, first + c * 16 + col, tile * kEach + r, v, w);
        }
    }
    order();
}
// Which rows a workgroup takes: item n of the first g.n is the first kChunk rows of run n, the items behind are long runs' further rows, kChunk each, so that a run which got most of the rows is
// gone through by many workgroups side by side (1024 rows in one of 64 experts 2048 x 768: 734 us one behind another, 80 so).  Where that makes many workgroups without rows, items are
// the chunks of all runs in order (listed): 2 rows among 32 experts 2880 x 2048 in codes 26.6 -> 18.6 us; the scan takes half a microsecond, 16 rows of eight 4096 x 1024 24.2 -> 25.2.
static __host__ __device__ __forceinline__ bool few_listed(int64_t n, int64_t n_rows, int64_t tiles) { return (n - n_rows) * tiles > 2048; }
template <int kChunk>
__device__ __forceinline__ bool few_chunk(const row_groups &g, int item, bool listed, int &e, int64_t &first, int &count)
{
    if (!listed && item < g.n) {
        int64_t end;
        e = item;
        group_bounds(g, e, first, end);
        count = (int)min(end - first, (int64_t)kChunk);
        return count > 0;
    }
    const uint32_t want = (uint32_t)(listed ? item : item - g.n);
    uint32_t before = 0;
    for (int c = 0; c < g.n; c += 64) {
        const int lane = (int)(threadIdx.x & 63);
        int64_t f = 0, end = 0;
        if (c + lane < g.n) group_bounds(g, c + lane, f, end);
        const int rows = (int)(end - f);
        const uint32_t chunks = (uint32_t)((rows + kChunk - 1) / kChunk) - (!listed && rows > 0), incl = before + mw_wave_incl_scan(chunks);
        const uint64_t behind = __ballot(incl > want);
        if (behind == 0) {
            before = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
            continue;
        }
        const int l = __ffsll((unsigned long long)behind) - 1;
        const int skip = (int)(want - (uint32_t)__builtin_amdgcn_readlane((int)(incl - chunks), l) + (listed ? 0 : 1)) * kChunk;
        e = c + l;
        first = __builtin_amdgcn_readlane((int)f, l) + skip;    // (rows are fewer than 2^31)
        count = min(__builtin_amdgcn_readlane(rows, l) - skip, kChunk);
        return true;
    }
    return false;
}
// A workgroup's kAlong waves share a tile of sixteen matrix rows, or (kAlong 1) each of four has its own.  grid: (tiles, four of them at kAlong 1; items, 65535 at most)
template <class Op, int kAlong>
__global__ __launch_bounds__(kAlong == 8 ? 512 : 256) void k_few(typename Op::args a)
{
    __shared__ __align__(16) char all[(kAlong == 8 ? 8 : 4) * 3 * kTileBytes];
    const int own = kAlong > 1 ? 0 : __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), tile = kAlong > 1 ? (int)blockIdx.x : (int)blockIdx.x * 4 + own;
    char *lds = all + own * 3 * kTileBytes;
    constexpr int kPass = 16 / Op::kTerms;
    const bool listed = few_listed(a.g.n, a.g.n_rows, (int64_t)gridDim.x * (kAlong > 1 ? 1 : 4));
    const int items = (int)(listed ? a.g.n_rows : a.g.n) + (int)(a.g.n_rows / (2 * kPass));
    for (int item = (int)blockIdx.y; item < items; item += (int)gridDim.y) {
        int e, count;
        int64_t first;
        if (!few_chunk<2 * kPass>(a.g, item, listed, e, first, count)) continue;
        e = __builtin_amdgcn_readfirstlane(e);                  // (the same for all lanes; said, so that arrays' places stay in scalar registers)
        count = __builtin_amdgcn_readfirstlane(count);
        first = __builtin_amdgcn_readfirstlane((int)first);
        if (count <= kPass) few_columns<Op, kAlong, 1, 4>(a, e, tile, first, count, lds);
        else few_columns<Op, kAlong, 2, 3>(a, e, tile, first, count, lds);
    }
}
// Waves that share sixteen matrix rows, by the tiles of all runs and the rows' bytes: eight where there is hardly a tile a CU and rows are long, one where there are many tiles of
// short rows, else four.  us of the call, one / four / eight:
//   1 row of four experts 7168 x 2048 23.7 / 24.3 / 20.7, of codes 7168 -> 4096 12.4 / 12.5 / 11.1 (256 tiles of 14336 and 7168 bytes)
//   second product, 64 rows of eight experts 4096 x 1024 (2048 tiles, 2048 bytes) 40.8 / 42.2 / 49.4, codes (1024 bytes) 27.8 / 32.3 / 41.5; 32 rows of four 7168 x 2048 (1792, 4096 bytes)
//   61.6 / 64.6 / 67.0; 32 rows of 32 experts 256 x 512 (512, 1024 bytes) 10.2 / 13.8 / 22.6; but 1 row of eight 4096 x 1024 (256, 2048 bytes) 14.4 / 11.9 / 14.0
//   64 rows of codes, eight matrices 4096 -> 1024 (512, 4096 bytes) 11.7 / 7.1 / 7.9, sixteen 2048 -> 768 (768, 2048 bytes) 7.2 / 5.5 / 10.3
static inline int few_waves(int64_t tiles, int64_t row_bytes)
{
    if (tiles <= 256 && row_bytes >= 4096) return 8;
    return (row_bytes <= 1024 && tiles >= 512) || (row_bytes <= 4096 && tiles >= 1792) ? 1 : 4;
}
template <class Op>
int32_t launch_few(const typename Op::args &a, int columns, hipStream_t s)
{
    const uint32_t tiles = (uint32_t)((columns + (Op::kPair ? 7 : 15)) / (Op::kPair ? 8 : 16));
    const int waves = few_waves((int64_t)tiles * (a.g.n < a.g.n_rows ? a.g.n : a.g.n_rows), (int64_t)a.K * (Op::kInt8 ? 1 : 2));
    const int64_t items = (few_listed(a.g.n, a.g.n_rows, waves > 1 ? tiles : (tiles + 3) / 4 * 4) ? a.g.n_rows : a.g.n) + a.g.n_rows / (32 / Op::kTerms);
    const uint32_t n = (uint32_t)(items < 65535 ? items : 65535);
    if (waves == 8) hipLaunchKernelGGL((k_few<Op, 8>), dim3(tiles, n), dim3(512), 0, s, a);
    else if (waves == 4) hipLaunchKernelGGL((k_few<Op, 4>), dim3(tiles, n), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_few<Op, 1>), dim3((tiles + 3) / 4, n), dim3(256), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    return MW_OK;
}

// How a product of rows with n matrices, `columns` values of a row from each, is cut: few rows a run to a form of their own, others to the tile size that is through first, counted
// in rounds of the CUs times what a step takes with a tile on every CU, 128 x 64, 256 x 128, 256 x 256 as 0.49 : 1 : 1.5 (fitted to 109
// calls of random sizes, each timed with all nine pairs of sizes for its two products: the sizes taken are 0.4 % from the best of them on average, 12 % at most).  parts: a last round's tiles
// may be cut along the sum.  us, weights from memory, runs of uneven lengths, both products with 128 x 64 / 256 x 128 / 256 x 256 tiles, and the ones taken:
//   mw_ffn, four experts 7168 x 2048, 512 rows 150 / 116 / 134, 123; 16384 rows - / - / 1242, the same; mw_ffn of codes, 512 rows 90 / 87 / 97, 90; 16384 rows 1062 / 854 / 804, 804
//   mw_ffn_backward, 333 rows of five 2880 x 1000 77 / 98 / 130, 77; 2048 rows of eight 4096 x 1024 209 / 203 / 195, 195
//   mw_matmul_int8, 8192 rows 7168 -> 7168 568 / 427 / 396, 396; four matrices 7168 -> 2048, 2048 rows 40 / 42 / 66, 40
// A few rows a run, 16 at most, with two terms a row (bf16 rows of h) 10 where the matrices make more tiles of 128 x 64 than there are CUs: mw_ffn, uneven runs, few / 128 x 64: four experts 7168 x 2048,
// 32 rows 67 / 87, 64 rows 84 / 88, 96 rows (even) 104 / 88; 32 of 4096 x 1024, 128 rows 128 / 153, 256 rows 140 / 154, 384 rows 157 / 153, 512 rows 181 / 154; codes, 512 rows 96 / 98;
// mw_matmul_int8, 64 matrices 4096 -> 1024, 1024 rows 58 / 62.
enum { kFew, kSmall, kMiddle, kLarge };
static inline double tile_rounds(int64_t n_rows, int64_t n, int rows_a_tile, int64_t column_tiles, int64_t at_once, int64_t steps, bool parts)
{
    const int64_t rows_tiles = (n_rows + rows_a_tile - 1) / rows_a_tile + (n - 1) / 2, runs = n < n_rows ? n : n_rows;         // (half of a run's last tile is empty)
    const int64_t tiles = (rows_tiles > runs ? rows_tiles : runs) * column_tiles, left = tiles % at_once, whole = (tiles - left) / kUnits;
    if (parts && left > 0 && parts_pay((uint32_t)left, (uint32_t)steps)) return (double)whole + (double)left / kUnits + (double)join_steps((uint32_t)left) / (double)steps;
    return (double)(whole + (left + kUnits - 1) / kUnits);
}
static inline int rows_form(int64_t n_rows, int64_t n, int64_t columns, int64_t steps, bool parts, int few = 16)
{
    if (n_rows <= few * n) return kFew;
    const double small = 0.49 * tile_rounds(n_rows, n, 64, (columns + 127) / 128, 512, steps, parts), middle = tile_rounds(n_rows, n, 128, (columns + 255) / 256, kUnits, steps, parts),
                 large = 1.5 * tile_rounds(n_rows, n, 256, (columns + 255) / 256, kUnits, steps, parts);
    return small < middle && small < large ? kSmall : middle < large ? kMiddle : kLarge;
}
// The forms of mw_ffn's two products (both have few rows or neither has), of mw_ffn_backward's da and dx (kFew: the smallest tiles), and of a product of codes.
struct two_forms { int first, second; };
static inline two_forms forward_forms(int64_t n_rows, int64_t n, int64_t hidden, int64_t inter)
{
    const int few = (2 * inter + 127) / 128 * n > kUnits ? 10 : 16;
    return {rows_form(n_rows, n, 2 * inter, (hidden + 63) / 64, true, few), rows_form(n_rows, n, hidden, (inter + 63) / 64, true, few)};
}
static inline two_forms backward_forms(int64_t n_rows, int64_t n, int64_t hidden, int64_t inter)
{
    return {rows_form(n_rows, n, inter, (hidden + 63) / 64, true), rows_form(n_rows, n, hidden, (2 * inter + 63) / 64, true)};
}
static inline int int8_form(int64_t n_rows, int64_t n, int64_t columns, int64_t n_in, bool parts) { return rows_form(n_rows, n, columns, (n_in + 127) / 128, parts); }
// Gradients of matrices by the runs' length and the tiles: sums of a few steps take 128 x 128 with room for one step, long ones over enough tiles 256 x 256.  us of k_ffn_grads without dx before it,
// medians of a kernel trace, uneven runs, 128 x 128 / 256 x 256: four experts 7168 x 2048, 512 rows 113 / 140, 2048 245 / 248, 4096 391 / 378, 8192 715 / 647, 16384 1565 / 1187; eight
// 4096 x 1024, 512 rows 44 / 62, 2048 85 / 93, 4096 132 / 130, 8192 226 / 210; 32 of 2048 x 768, 4096 rows 94 / 116; five 2880 x 1000, 333 rows 27 / 33, 2000 56 / 57; two 1024 x 512 (48 of
// the larger tiles), 4000 rows 48 / 54.
static inline bool grads_large(int64_t n_rows, int64_t n, int64_t hidden, int64_t inter)
{
    return n_rows >= 512 * n && ((2 * inter + 255) / 256 + (inter + 255) / 256) * ((hidden + 255) / 256) * n >= kUnits;
}
// The tile sizes' arguments are alike.
template <class To, class From> To as(const From &f)
{
    static_assert(sizeof(To) == sizeof(From), "");
    return __builtin_bit_cast(To, f);
}
// Large, Middle, Small: one product with tiles of 256 x 256, 256 x 128 and 128 x 64.  kHasFew: the product has few_emit().
template <class Large, class Middle, class Small, bool kHasFew>
int32_t launch_product(int form, const typename Large::args &a, int columns, hipStream_t s)
{
    if constexpr (kHasFew) if (form == kFew) return launch_few<Large>(a, columns, s);
    if (form == kLarge) return launch_tiles<Large>(a, columns, s);
    if (form == kMiddle) return launch_tiles<Middle>(as<typename Middle::args>(a), columns, s);
    return launch_tiles<Small>(as<typename Small::args>(a), columns, s);
}

}  // namespace
#endif  // MW_FEW_H_
