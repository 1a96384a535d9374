// Products of tiles that stay in registers: the experts' products over many rows.
//
// A workgroup of four waves makes a tile of kP columns times kQ rows of an output, one wave a quarter of it, kP / 2 by kQ / 2, in the accumulators
// of 32 x 32 matrix instructions.  Steps of 128 bytes along the sum (64 bf16 values, 128 codes) come from memory straight into LDS, two steps' room; a step's
// four parts go from LDS to registers one ahead of the instructions that use them.  The matrix instruction's first operand is the tile of columns (weights), so a
// lane's results are neighbours in a row of the output.
//
// LDS holds an operand as it comes, a kilobyte a load and wave, so places change only with what each lane asks for.  Where the sum runs along the
// operand's rows, a row is 128 bytes and its 16-byte chunks are exchanged by the row's number (chunk ^ row % 8): eight lanes of a read are on different banks.  Where it runs
// across them (kTr), 64 lines of kR values are there, a line's 32-byte chunks exchanged by the line's number, and a read that transposes four lines of sixteen values makes
// the operand.
#ifndef MW_TILE_H_
#define MW_TILE_H_

#include "mw_math.h"

namespace {

typedef __amdgpu_buffer_rsrc_t tile_array;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
constexpr uint32_t kNowhereAt = 0x80000000u;

constexpr int kTileWaves = 4, kTileThreads = 64 * kTileWaves;
constexpr int kStep = 128;               // bytes along the sum of a step

template <bool kInt8> struct tile_kind;
template <> struct tile_kind<false> {
    typedef bf16x8 frag; typedef f32x16 acc; static constexpr int bytes = 2;
    static __device__ __forceinline__ acc mma(frag a, frag b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct tile_kind<true> {
    typedef i32x4 frag; typedef i32x16 acc; static constexpr int bytes = 1;
    static __device__ __forceinline__ acc mma(frag a, frag b, acc c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};

// 16 bytes a lane from memory to LDS, the wave's kilobyte in lane order; kNowhereAt: zeros.  (The host's pass does not know these two instructions.)
__device__ __forceinline__ void load_to_lds(tile_array from, lds_char *to, uint32_t at)
{
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, at, 0, 0, 0);
#endif
}
// Four values each of sixteen lanes, a row of sixteen to every four lanes -> every lane has its column's four.
__device__ __forceinline__ s16x4 read_transposed(lds_char *p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
#else
    return s16x4{};
#endif
}

template <int kR, bool kTr, bool kInt8>
struct tile_feed {
    static constexpr int kPieces = kR / 32, kBytes = kR * kStep;
    static constexpr int kLines = 512 / kR;                     // kTr: rows of a piece
    const char *base;
    int64_t step;
    int limit;                                                  // K
    int lane_k;
    uint32_t at[kPieces];
    // kTr == false: place(r) gives the byte of row r of the tile, or kNowhereAt
    template <class F>
    __device__ __forceinline__ void rows(const char *from, int k, F place)
    {
        static_assert(!kTr, "");
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        base = from; step = kStep; limit = k;
        const int chunk = (lane & 7) ^ (lane >> 3);
        lane_k = chunk * (kInt8 ? 16 : 8);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const uint32_t p = place((j * kTileWaves + wave) * 8 + (lane >> 3));
            at[j] = p == kNowhereAt ? p : p + (uint32_t)chunk * 16;
        }
    }
    __device__ __forceinline__ void lines(const char *from, int k, int64_t stride_bytes, int width)
    {
        static_assert(kTr && !kInt8, "");
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        base = from; step = 64 * stride_bytes; limit = k;
        lane_k = wave * kLines + lane / (kR / 8);
        const int u = lane % (kR / 8);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int kk = lane_k + j * kTileWaves * kLines, s = ((kk & 3) | ((kk >> 3) & 1) << 2) & (kR / 16 - 1);
            const int mn = ((u >> 1) ^ s) * 16 + (u & 1) * 8;
            at[j] = mn < width ? (uint32_t)kk * (uint32_t)stride_bytes + 2u * (uint32_t)mn : kNowhereAt;
        }
    }
    // What step k's loads share, and one of them (of kPieces).
    struct step_of { tile_array r; int left; lds_char *to; };
    __device__ __forceinline__ step_of at_step(int k, lds_char *to) const
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        return step_of{__builtin_amdgcn_make_buffer_rsrc((void *)(base + (int64_t)k * step), 0, (int)kNowhereAt, 0x00027000),
                       limit - k * (kTr ? 64 : kStep / (kInt8 ? 1 : 2)), to + wave * 1024};
    }
    __device__ __forceinline__ void issue(const step_of &s, int j) const
    {
        const uint32_t off = lane_k < s.left - (kTr ? j * kTileWaves * kLines : 0) ? at[j] : kNowhereAt;
        load_to_lds(s.r, s.to + j * kTileWaves * 1024, off);
    }
    __device__ __forceinline__ void issue_all(int k, lds_char *to) const
    {
        const step_of s = at_step(k, to);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) issue(s, j);
    }
};

// A wave's half of one operand in the stage: kN pieces of 32 rows, four steps of 16 (32 codes) along K.
template <int kR, bool kTr, bool kInt8>
struct tile_frags {
    typedef typename tile_kind<kInt8>::frag frag;
    static constexpr int kN = kR / 64;
    uint32_t from[4];
    __device__ __forceinline__ void begin(int half)
    {
        const int lane = threadIdx.x & 63;
        if constexpr (!kTr) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) from[kk] = (uint32_t)(half * (kR / 2) + (lane & 31)) * kStep + (((kk * 2 + (lane >> 5)) ^ (lane & 7)) * 16);
        } else {
            // sixteen lanes take four rows of 16 values: row (lane / 4) % 4, values (lane % 4) * 4 ..; the rows' 32-byte chunks change places with the row
            const int k = (lane >> 5) * 8 + ((lane >> 2) & 3), chunk = half * (kR / 32) + ((lane >> 4) & 1);
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                // (k + 4 and k + 16 have the same two bits: one place for each of the piece's two reads and of the four steps)
                const int s = ((k & 3) | ((k >> 3) & 1) << 2) & (kR / 16 - 1);
                from[kk] = (uint32_t)(k * kR * 2 + (chunk ^ s) * 32 + (lane & 3) * 8);
            }
        }
    }
    __device__ __forceinline__ frag read(const lds_char *stage, int kk, int t) const
    {
        if constexpr (!kTr) {
            return *(const __attribute__((address_space(3))) frag *)(stage + from[kk] + t * 32 * kStep);
        } else {
            lds_char *p = (lds_char *)stage + (from[0] ^ (uint32_t)(t * 64)) + kk * 16 * kR * 2;
            return __builtin_bit_cast(frag, __builtin_shufflevector(read_transposed(p), read_transposed(p + 4 * kR * 2), 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

__device__ __forceinline__ void tile_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
template <int kN> __device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt((kN & 15) | (kN >> 4) << 14 | 0x0f70); }

// kN times: one read of LDS, kM matrix instructions; whatever is left of them after that.
template <int kReads, int kLoads, int kMfma>
__device__ __forceinline__ void tile_mix()
{
#pragma unroll
    for (int n = 0; n < kMfma; ++n) {
        if (n < kLoads) __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
        if (n < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
}
template <int kP, int kQ, bool kTrP, bool kTrQ, bool kInt8>
struct tile_product {
    typedef tile_kind<kInt8> kind;
    typedef typename kind::frag frag;
    static constexpr int kNP = kP / 64, kNQ = kQ / 64, kStage = (kP + kQ) * kStep, kLds = 2 * kStage, kLoads = (kP + kQ) / 32;
    typename kind::acc acc[kNP][kNQ];
    __device__ __forceinline__ void run(const tile_feed<kP, kTrP, kInt8> &p, const tile_feed<kQ, kTrQ, kInt8> &q, int steps, lds_char *lds)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        tile_frags<kP, kTrP, kInt8> fp;
        tile_frags<kQ, kTrQ, kInt8> fq;
        fp.begin(wave & 1);
        fq.begin(wave >> 1);
        frag a[2][kNP], b[2][kNQ];
        auto read = [&](int set, const lds_char *stage, int kk, int n) {
            if (n < kNP) a[set][n] = fp.read(stage, kk, n);
            else b[set][n - kNP] = fq.read(stage + kP * kStep, kk, n - kNP);
        };
        auto multiply = [&](int set, int n) {
            const int i = n / kNQ, j = n % kNQ;
            acc[i][j] = kind::mma(a[set][i], b[set][j], acc[i][j]);
        };
        constexpr int kReads = kNP + kNQ, kMfma = kNP * kNQ, kInstr = kNP * (kTrP ? 2 : 1) + kNQ * (kTrQ ? 2 : 1);
#pragma unroll
        for (int n = 0; n < kMfma; ++n) acc[n / kNQ][n % kNQ] = typename kind::acc{};
        p.issue_all(0, lds); q.issue_all(0, lds + kP * kStep);
        p.issue_all(1, lds + kStage); q.issue_all(1, lds + kStage + kP * kStep);
        wait_loads<kLoads>();
        tile_barrier();
#pragma unroll
        for (int n = 0; n < kReads; ++n) read(0, lds, 0, n);
        for (int k = 0; k < steps; ++k) {
            lds_char *here = lds + (k & 1) * kStage, *next = lds + ((k + 1) & 1) * kStage;
#pragma unroll
            for (int kk = 0; kk < 3; ++kk) {
#pragma unroll
                for (int n = 0; n < kReads; ++n) read((kk + 1) & 1, here, kk + 1, n);
#pragma unroll
                for (int n = 0; n < kMfma; ++n) multiply(kk & 1, n);
                tile_mix<kInstr, 0, kMfma>();
            }
            __builtin_amdgcn_s_waitcnt(0x0070);         // this wave has read its last of this stage, and its part of the next one is there
            tile_barrier();
            const auto sp = p.at_step(k + 2, here);
            const auto sq = q.at_step(k + 2, here + kP * kStep);
            constexpr int kSlots = kLoads > kMfma ? kLoads : kMfma;
#pragma unroll
            for (int n = 0; n < kSlots; ++n) {
                if (n < kReads) read(0, next, 0, n);
                if (n < kP / 32) p.issue(sp, n);
                else if (n < kLoads) q.issue(sq, n - kP / 32);
                if (n < kMfma) multiply(1, n);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        wait_loads<0>();
    }
};

// ---- rows in runs, one run a matrix ---------------------------------------------------------------------------
struct row_groups {
    const int64_t *offsets;     // [n + 1], or null: one run of all rows
    int64_t n_rows;
    int32_t n;
};
__device__ __forceinline__ void group_bounds(const row_groups &g, int e, int64_t &first, int64_t &end)
{
    if (!g.offsets) { first = 0; end = g.n_rows; return; }
    first = min(max(g.offsets[e], (int64_t)0), g.n_rows);
    end = min(max(g.offsets[e + 1], first), g.n_rows);
}
struct tile_at {
    int e;                      // run
    int64_t first;              // first row of the tile
    int rows;                   // rows of the run from there on (at least one)
    int p;                      // tile of columns
};
// Runs of consecutive tiles go to one of the eight XCDs each, whose L2 then holds what they share.  Workgroups are dealt out to XCDs in turn.
__device__ __forceinline__ bool tile_of_workgroup(uint32_t total, uint32_t &t)
{
    const uint32_t per = (total + 7) / 8, at = blockIdx.x >> 3;
    t = (blockIdx.x & 7) * per + at;
    return at < per && t < total;
}
// Inside a run (or matrix) tiles go down kBlock tiles of rows before the next tile of columns.
constexpr uint32_t kBlock = 8;
__device__ __forceinline__ void tile_in_block(uint32_t t, uint32_t p_tiles, uint32_t q_tiles, uint32_t &p, uint32_t &q)
{
    const uint32_t block = t / (kBlock * p_tiles), left = t - block * kBlock * p_tiles, high = min(kBlock, q_tiles - block * kBlock);
    p = left / high;
    q = block * kBlock + left % high;
}
template <int kQ>
__device__ __forceinline__ bool find_tile(const row_groups &g, uint32_t p_tiles, tile_at &at)
{
    const int lane = threadIdx.x & 63;
    int64_t first = 0, end = 0;
    if (lane < g.n) group_bounds(g, lane, first, end);
    uint32_t tiles = (uint32_t)((end - first + kQ - 1) / kQ), total = mw_wave_sum(tiles);
    for (int c = 64; c < g.n; c += 64) {
        int64_t f = 0, l = 0;
        if (c + lane < g.n) group_bounds(g, c + lane, f, l);
        total += mw_wave_sum((uint32_t)((l - f + kQ - 1) / kQ));
    }
    uint32_t t;
    if (!tile_of_workgroup(total * p_tiles, t)) return false;
    uint32_t before = 0;
    const uint32_t want = t / p_tiles;
    for (int c = 0;; c += 64) {
        if (c > 0) {
            first = end = 0;
            if (c + lane < g.n) group_bounds(g, c + lane, first, end);
            tiles = (uint32_t)((end - first + kQ - 1) / kQ);
        }
        const uint32_t incl = before + mw_wave_incl_scan(tiles);
        const uint64_t behind = __ballot(incl > want);
        if (behind == 0) {
            before = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
            continue;
        }
        const int l = __ffsll((unsigned long long)behind) - 1;
        const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)tiles, l), start = (uint32_t)__builtin_amdgcn_readlane((int)incl, l) - mine;
        const int64_t f = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)first, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(first >> 32), l) << 32);
        const int rows = __builtin_amdgcn_readlane((int)(end - first), l);
        uint32_t p, q;
        tile_in_block(t - start * p_tiles, p_tiles, mine, p, q);
        at.e = c + l; at.first = f + (int64_t)q * kQ; at.rows = rows - (int)q * kQ; at.p = (int)p;
        return true;
    }
}
static inline int64_t most_tiles(int64_t n_rows, int64_t n, int rows_a_tile) { return n_rows / rows_a_tile + (n < n_rows ? n : n_rows); }
// Workgroups of a launch for `tiles` tiles; 0: too many.
static inline uint32_t tile_grid(int64_t tiles) { return tiles > 0x7ffffff0LL ? 0u : (uint32_t)((tiles + 7) / 8 * 8); }

// Row r of a tile of columns in LDS -> column of the tile: lanes then hold sixteen columns in a row of each 32 (the matrix instruction's result
// has eights of rows, the lower four of each in the lower half of the wave).
__device__ __forceinline__ int tile_column(int r) { return (r & ~31) | ((r >> 2) & 1) << 4 | ((r >> 3) & 3) << 2 | (r & 3); }

__device__ __forceinline__ float tile_sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }
template <int kN>
__device__ __forceinline__ void store_bf16(uint16_t *to, const float *v)
{
    static_assert(kN == 4 || kN == 8, "");
    typedef __bf16 vec __attribute__((ext_vector_type(kN)));
    vec o;
#pragma unroll
    for (int i = 0; i < kN; ++i) o[i] = (__bf16)v[i];
    *(vec *)to = o;
}

}  // namespace
#endif  // MW_TILE_H_
