// Products of tiles that stay in registers: the experts' products over many rows.
//
// A workgroup of four waves makes a tile of kP columns times kQ rows of an output, one wave a quarter of it, kP / 2 by kQ / 2, in the accumulators
// of 32 x 32 matrix instructions.  Steps of 128 bytes along the sum (64 bf16 values, 128 codes) come from memory straight into LDS, two steps' room (tiles of 128 x 64 three).  A step's
// first quarter is in registers when the step begins; beside its products the other three come from LDS, then the stage is free and the step after the next is loaded into
// it while two more quarters are multiplied, and beside the last one the next step's first quarter comes.  A load has four fifths of two steps
// to arrive that way; with the stage free only after a step's last quarter had been read it had two fifths: 16384 x 4096, sums of 7168, 795 us instead of 740 (columns by
// lines), 8192^3 867 instead of 792.  The matrix instruction's first operand is the tile of columns (weights), so a lane's results are neighbours in a row of the output.
//
// LDS holds an operand as it comes, a kilobyte a load and wave, so places change only with what each lane asks for.  Where the sum runs along the
// operand's rows, a row is 128 bytes and its 16-byte chunks are exchanged by the row's number: a read of 32 rows uses all banks evenly.  Where it runs
// across them (kTr), 64 lines of kR values are there, a line's 32-byte chunks exchanged by the line's number, and a read that transposes four lines of sixteen values makes
// the operand.  Neither has a bank conflict (counted).
//
// What bounds it: with all CUs busy the matrix instructions and, behind them, the clock that the card holds while they run (a large product's first calls after a pause take a tenth less than
// those that follow).  16384 rows of codes times 7168 x 7168, 757 us (least 688), 2220 TOP/s (2450); bf16 sums of 7168, 16384 x 4096, 750 us (720), 1280 TFLOP/s (1340); 10 to 18 us a round of tiles go to first loads and to results.
// Workgroups that stay, and load their next tile's first step before the results of the one before leave, were not faster (sums of 7168 and 2048, 16384 rows, 1240 -> 1246 us; gradients
// of uneven runs 2429 -> 2526): the hardware hands the next tile to whichever CU is free.
#ifndef MW_TILE_H_
#define MW_TILE_H_

#include "mw_stream.h"

namespace {

typedef u32x4 tile_array;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
struct tile_nothing {};
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;
constexpr uint32_t kNowhereAt = 0x80000000u;

constexpr int kTileWaves = 4, kTileThreads = 64 * kTileWaves;
constexpr int kStep = 128;               // bytes along the sum of a step

template <bool kInt8> struct tile_kind;
template <> struct tile_kind<false> {
    typedef bf16x8 frag; typedef f32x16 acc;
    static __device__ __forceinline__ acc mma(frag a, frag b, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct tile_kind<true> {
    typedef i32x4 frag; typedef i32x16 acc;
    static __device__ __forceinline__ acc mma(frag a, frag b, acc c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};

__device__ __forceinline__ int exchange(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int exchange_lines(int line) { return (line & 3) << 1; }

// An array of 2 GiB whose loads past its end are zeros and cost no traffic.
__device__ __forceinline__ tile_array tile_array_at(const char *p)
{
    const uint64_t a = (uint64_t)p;
    return tile_array{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)) & 0xffffu, kNowhereAt, 0x00027000u};
}
// 16 bytes a lane from memory to LDS, the wave's kilobyte in lane order; kNowhereAt: zeros.  Written out, because the compiler lets a transposing read wait
// for every such load on the way, whichever part of LDS it goes to.  It has no result in registers; who reads what it brings waits with tile_wait.
// M0 is used for nothing else in these kernels.
__device__ __forceinline__ void load_to_lds(tile_array from, lds_char *to, uint32_t at)
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"((uint32_t)(uintptr_t)to), "v"(at), "s"(from) : "memory");
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
    int piece0;                                                 // byte of the wave's first piece
    uint32_t at[kPieces];
    // kTr == false: place(r) gives the byte of row r of the tile, or kNowhereAt
    template <class F>
    __device__ __forceinline__ void rows(const char *from, int k, F place)
    {
        static_assert(!kTr, "");
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        base = from; step = kStep; limit = k; piece0 = wave * 1024;
        const int chunk = (lane & 7) ^ exchange((wave & 1) * 8 + (lane >> 3));
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
        base = from; step = 64 * stride_bytes; limit = k; piece0 = wave * 1024;
        lane_k = wave * kLines + lane / (kR / 8);
        const int u = lane % (kR / 8);
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            const int kk = lane_k + j * kTileWaves * kLines, s = exchange_lines(kk) & (kR / 16 - 1);
            const int mn = ((u >> 1) ^ s) * 16 + (u & 1) * 8;
            at[j] = mn < width ? (uint32_t)kk * (uint32_t)stride_bytes + 2u * (uint32_t)mn : kNowhereAt;
        }
    }
    // Steps first .. first + n - 1 only.
    __device__ __forceinline__ void part(int first, int n)
    {
        constexpr int kEach = kTr ? 64 : kStep / (kInt8 ? 1 : 2);
        base += (int64_t)first * step;
        limit = min(limit - first * kEach, n * kEach);
    }
    // What step k's loads share, and one of them (of kPieces).
    struct step_of { tile_array r; int left; lds_char *to; };
    __device__ __forceinline__ step_of at_step(int k, lds_char *to) const
    {
        return step_of{tile_array_at(base + (int64_t)k * step),
                       limit - k * (kTr ? 64 : kStep / (kInt8 ? 1 : 2)), to + piece0};
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
    uint32_t from[kTr ? 1 : 4];
    __device__ __forceinline__ void begin(int half)
    {
        const int lane = threadIdx.x & 63;
        if constexpr (!kTr) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) from[kk] = (uint32_t)(half * (kR / 2) + (lane & 31)) * kStep + (((kk * 2 + (lane >> 5)) ^ exchange(lane & 15)) * 16);
        } else {
            // sixteen lanes take four rows of 16 values: row (lane / 4) % 4, values (lane % 4) * 4 ..; the rows' 32-byte chunks change places with the row.  One place serves the piece's two
            // reads (rows k and k + 4) and the four steps along K (16 rows on): these rows' lowest two bits, by which chunks change places, are k's.
            const int k = (lane >> 5) * 8 + ((lane >> 2) & 3), chunk = half * (kR / 32) + ((lane >> 4) & 1), s = exchange_lines(k) & (kR / 16 - 1);
            from[0] = (uint32_t)(k * kR * 2 + (chunk ^ s) * 32 + (lane & 3) * 8);
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
// Until at most kN of this wave's loads are on the way; kReads: and all its reads of LDS are done.
template <int kN, bool kReads = false>
__device__ __forceinline__ void tile_wait()
{
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (kReads) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(kN) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kN) : "memory");
#endif
}

__device__ __forceinline__ void tile_reads_done()
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
#endif
    tile_barrier();
}

template <int kP, int kQ, bool kTrP, bool kTrQ, bool kInt8>
struct tile_product {
    typedef tile_kind<kInt8> kind;
    typedef typename kind::frag frag;
    static constexpr int kNP = kP / 64, kNQ = kQ / 64, kStages = kP * kQ == 128 * 64 ? 3 : 2, kStage = (kP + kQ) * kStep, kLds = kStages * kStage, kLoads = (kP + kQ) / 32;
    typename kind::acc acc[kNP][kNQ];
    __device__ __forceinline__ void run(const tile_feed<kP, kTrP, kInt8> &p, const tile_feed<kQ, kTrQ, kInt8> &q, int steps, lds_char *lds)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        tile_frags<kP, kTrP, kInt8> fp;
        tile_frags<kQ, kTrQ, kInt8> fq;
        fp.begin(wave & 1);
        fq.begin(wave >> 1);
        frag a[4][kNP], b[4][kNQ];
        auto read = [&](const lds_char *stage, int kk, int n) {
            if (n < kNP) a[kk][n] = fp.read(stage, kk, n);
            else b[kk][n - kNP] = fq.read(stage + kP * kStep, kk, n - kNP);
        };
        auto multiply = [&](int kk, int n) {
            const int i = n / kNQ, j = n % kNQ;
            acc[i][j] = kind::mma(a[kk][i], b[kk][j], acc[i][j]);
        };
        constexpr int kReads = kNP + kNQ, kMfma = kNP * kNQ;
#pragma unroll
        for (int n = 0; n < kMfma; ++n) acc[n / kNQ][n % kNQ] = typename kind::acc{};
#pragma unroll
        for (int k = 0; k < kStages; ++k) { p.issue_all(k, lds + k * kStage); q.issue_all(k, lds + k * kStage + kP * kStep); }
        tile_wait<(kStages - 1) * kLoads>();
        tile_barrier();
#pragma unroll
        for (int n = 0; n < kReads; ++n) read(lds, 0, n);
        lds_char *here = lds;
        for (int k = 0; k < steps; ++k) {
            lds_char *next = here == lds + (kStages - 1) * kStage ? lds : here + kStage;
            // the step's other three parts come to registers beside the first part's products, in the first three quarters of them
            constexpr int kEarly = (kMfma * 3 + 3) / 4;
#pragma unroll
            for (int n = 0; n < kMfma; ++n) {
#pragma unroll
                for (int r = n * 3 * kReads / kEarly; r < (n + 1) * 3 * kReads / kEarly; ++r)
                    if (r < 3 * kReads) read(here, 1 + r / kReads, r % kReads);
                multiply(0, n);
                __builtin_amdgcn_sched_barrier(0);
            }
            tile_reads_done();                          // every wave has read this stage: it is loaded again, for step k + kStages
            const auto sp = p.at_step(k + kStages, here);
            const auto sq = q.at_step(k + kStages, here + kP * kStep);
#pragma unroll
            for (int n = 0; n < 2 * kMfma; ++n) {
#pragma unroll
                for (int l = n * kLoads / (2 * kMfma); l < (n + 1) * kLoads / (2 * kMfma); ++l) {
                    if (l < kP / 32) p.issue(sp, l);
                    else q.issue(sq, l - kP / 32);
                }
                multiply(1 + n / kMfma, n % kMfma);
                __builtin_amdgcn_sched_barrier(0);
            }
            tile_wait<(kStages - 1) * kLoads>();        // the next step's loads, every wave's
            tile_barrier();
#pragma unroll
            for (int n = 0; n < kMfma; ++n) {
#pragma unroll
                for (int r = n * kReads / kEarly; r < (n + 1) * kReads / kEarly; ++r)
                    if (r < kReads) read(next, 0, r);
                multiply(3, n);
                __builtin_amdgcn_sched_barrier(0);
            }
            here = next;
        }
        tile_wait<0>();
        tile_reads_done();                              // (the results go through LDS)
        stay();
    }
    // The accumulators stay where the matrix instructions left them until a piece is used: brought to ordinary registers together, they are spilled.
    __device__ __forceinline__ void stay()
    {
#if defined(__HIP_DEVICE_COMPILE__)
        if constexpr (kNP * kNQ == 16) {
#pragma unroll
            for (int n = 0; n < kNP * kNQ; ++n) asm volatile("" : "+a"(acc[n / kNQ][n % kNQ]));
        }
#endif
    }
};

// The same with room for one step: for sums of a few steps, whose time is waiting for the first loads and writing results, five workgroups a CU that wait for themselves hide
// more than two that load ahead.  us, room for two / one, medians of a kernel trace over uneven runs: gradients of 512 rows over eight experts 4096 x 1024 59 / 44, 2048 rows 103 / 85, four
// 7168 x 2048, 512 rows 146 / 113, 2048 rows 268 / 245.  Long sums over few tiles want the room: 4000 rows over two experts 1024 x 512 24 / 48; products of rows, mw_ffn, 512 rows of four
// 7168 x 2048 120 / 159, 16384 rows 1223 / 1807.
template <int kP, int kQ, bool kTrP, bool kTrQ, bool kInt8>
struct tile_product_short {
    typedef tile_kind<kInt8> kind;
    typedef typename kind::frag frag;
    static constexpr int kNP = kP / 64, kNQ = kQ / 64, kStage = (kP + kQ) * kStep, kLds = kStage;
    typename kind::acc acc[kNP][kNQ];
    __device__ __forceinline__ void run(const tile_feed<kP, kTrP, kInt8> &p, const tile_feed<kQ, kTrQ, kInt8> &q, int steps, lds_char *lds)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
        tile_frags<kP, kTrP, kInt8> fp;
        tile_frags<kQ, kTrQ, kInt8> fq;
        fp.begin(wave & 1);
        fq.begin(wave >> 1);
#pragma unroll
        for (int n = 0; n < kNP * kNQ; ++n) acc[n / kNQ][n % kNQ] = typename kind::acc{};
        for (int k = 0; k < steps; ++k) {
            p.issue_all(k, lds);
            q.issue_all(k, lds + kP * kStep);
            tile_wait<0>();
            tile_barrier();
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                frag a[kNP], b[kNQ];
#pragma unroll
                for (int i = 0; i < kNP; ++i) a[i] = fp.read(lds, kk, i);
#pragma unroll
                for (int j = 0; j < kNQ; ++j) b[j] = fq.read(lds + kP * kStep, kk, j);
#pragma unroll
                for (int n = 0; n < kNP * kNQ; ++n) acc[n / kNQ][n % kNQ] = kind::mma(a[n / kNQ], b[n % kNQ], acc[n / kNQ][n % kNQ]);
            }
            tile_reads_done();
        }
    }
};

// A launch has fewer than 2^32 threads along an axis (2^24 workgroups of kTileThreads): workgroups beyond kAcross go into further rows of the grid, which the hardware deals out like one long row.
constexpr uint32_t kAcross = 1u << 20;
__host__ __device__ __forceinline__ uint32_t rows_of_grid(uint32_t workgroups) { return (workgroups + kAcross - 1) / kAcross; }
static inline dim3 grid_of(uint32_t workgroups) { return dim3(workgroups < kAcross ? workgroups : kAcross, rows_of_grid(workgroups)); }
__device__ __forceinline__ uint32_t workgroup_id() { return blockIdx.y * kAcross + blockIdx.x; }

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
// Work is cut into units: a whole tile, or a part of a tile's sum.  kRound workgroups run at a time, so T tiles of one duration take ceil(T / kRound) rounds; the tiles of
// a last round may be cut into as many parts as fill it.  The parts' sums go to memory, and k_join adds them up in their order.
//
// That pays if it saves more steps than writing, reading and a launch cost, which is as many for all three tile sizes (a step of 128 x 64, 256 x 128 and 256 x 256 takes 0.33, 0.63 and
// 1.3 us, a join with its traffic 10, 20 and 41 us).  R tiles on 256 CUs leave 1 - R / 256 of them idle.  us of a call whole / in parts, its products' steps and tiles:
//   128 x 64: 128 rows of one expert 4096 x 2048 (64 steps of 64 tiles, 32 of 64) 40 / 33, 512 rows (256 tiles both) 43 / 58; 512 rows of four 7168 x 2048, backward without the
//   matrices' gradients (112 of 128, 64 of 448) 138 / 126, forward (112 of 256, 32 of 448) 104 / 113; 333 rows of five 2880 x 1000, backward (45 of 80, 32 of 230) 36 / 42
//   256 x 128: 512 rows of four 7168 x 2048 (112 of 64, 32 of 112) 149 / 99; 1024 rows of one 4096 x 2048 (64 of 128, 32 of 128) 70 / 80
//   256 x 256: 2048 rows of four 7168 x 2048 (112 of 128, 32 of 224) 221 / 188; 2048 rows of one 4096 x 2048 (64 of 128, 32 of 128) 115 / 134
constexpr uint32_t kMostParts = 16, kLeastSteps = 8, kUnits = 256;
__host__ __device__ __forceinline__ uint32_t join_steps(uint32_t tiles) { return 20 + tiles / 8; }
__host__ __device__ __forceinline__ bool parts_pay(uint32_t tiles, uint32_t steps) { return tiles < kUnits && (uint64_t)steps * (kUnits - tiles) >= (uint64_t)join_steps(tiles) * kUnits; }
struct tile_split { uint32_t whole, rest, parts; };             // tiles in one piece, tiles in parts, parts of each (1: rest are in one piece too)
__host__ __device__ __forceinline__ tile_split split_tiles(uint32_t total, uint32_t round, uint32_t steps, bool may)
{
    tile_split s = {total - total % round, total % round, 1};
    if (may && s.rest > 0 && parts_pay(s.rest, steps)) s.parts = max(1u, min(min(round / s.rest, kMostParts), steps / kLeastSteps));
    return s;
}
struct tile_unit { uint32_t tile, part; };
// Runs of consecutive units go to one of the eight XCDs each, whose L2 then holds what they share.  Workgroups are dealt out to XCDs in turn.
__device__ __forceinline__ bool unit_of_workgroup(const tile_split &s, tile_unit &u)
{
    uint32_t id = workgroup_id();
    const bool whole = id < s.whole;
    if (!whole) id -= s.whole;                                  // (a multiple of eight)
    const uint32_t n = whole ? s.whole : s.rest * s.parts, per = (n + 7) / 8, at = id >> 3, t = (id & 7) * per + at;
    if (at >= per || t >= n) return false;
    u.part = whole ? 0 : t / s.rest;
    u.tile = whole ? t : s.whole + t % s.rest;
    return true;
}
// Inside a run (or matrix) tiles go down kBlock tiles of rows before the next tile of columns.  us, 4 / 8 / 16: 8192^3 codes 465 / 600 / 704, bf16 805 / 816 / 865.
constexpr uint32_t kBlock = 4;
__device__ __forceinline__ void tile_in_block(uint32_t t, uint32_t p_tiles, uint32_t q_tiles, uint32_t &p, uint32_t &q)
{
    const uint32_t block = t / (kBlock * p_tiles), left = t - block * kBlock * p_tiles, high = min(kBlock, q_tiles - block * kBlock);
    p = left / high;
    q = block * kBlock + left % high;
}
// The runs' tiles of kQ rows, one run a lane; the first 64 stay in registers.
template <int kQ>
struct tile_runs {
    int64_t first, end;
    uint32_t tiles, total;
    __device__ __forceinline__ void load(const row_groups &g, int c)
    {
        const int e = c + (int)(threadIdx.x & 63);
        first = end = 0;
        if (e < g.n) group_bounds(g, e, first, end);
        tiles = (uint32_t)((end - first + kQ - 1) / kQ);
    }
    __device__ __forceinline__ void count(const row_groups &g)
    {
        total = 0;
        for (int c = (g.n - 1) / 64 * 64; c >= 0; c -= 64) {
            load(g, c);
            total += mw_wave_sum(tiles);
        }
    }
    // Tile t of p_tiles for each tile of rows, after count().
    __device__ __forceinline__ bool find(const row_groups &g, uint32_t p_tiles, uint32_t t, tile_at &at)
    {
        uint32_t before = 0;
        const uint32_t want = t / p_tiles;
        for (int c = 0; c < g.n; c += 64) {
            if (c > 0) load(g, c);
            const uint32_t incl = before + mw_wave_incl_scan(tiles);
            const uint64_t behind = __ballot(incl > want);
            if (behind == 0) {
                before = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
                continue;
            }
            const int l = __ffsll((unsigned long long)behind) - 1;
            const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)tiles, l), start = (uint32_t)__builtin_amdgcn_readlane((int)incl, l) - mine;
            const int64_t f = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)first, l) |
                                        (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(first >> 32), l) << 32);
            const int rows = __builtin_amdgcn_readlane((int)(end - first), l);
            uint32_t p, q;
            tile_in_block(t - start * p_tiles, p_tiles, mine, p, q);
            at.e = c + l; at.first = f + (int64_t)q * kQ; at.rows = rows - (int)q * kQ; at.p = (int)p;
            return true;
        }
        return false;
    }
};

// How results leave: a wave's quarter of a tile goes through LDS, 64 (small tiles: 32) rows at a time, and comes back eight neighbouring columns a lane, whole rows of it to
// neighbouring lanes: memory is written (and what belongs to the results is read) in whole lines.  From the accumulators a lane would write sixteen bytes here and there.
// kPair: the wave's columns are two halves that belong together, a lane gets eight of each.
template <int kP, int kQ, bool kPair>
struct tile_out {
    static constexpr int kCols = kP / 2, kRows = kP * kQ <= 128 * 128 ? 32 : 64, kPitch = kCols * 4 + 16, kBytes = kRows * kPitch;          // (rows begin on different banks)
    static constexpr int kLanes = kCols / (kPair ? 16 : 8), kAtOnce = 64 / kLanes;                                                      // lanes of a row, rows at once
    template <class Acc>
    static __device__ __forceinline__ void put(lds_char *lds, int i, int j, const Acc &v)                                              // piece i, j (of kRows / 32) of the accumulators
    {
        const int lane = threadIdx.x & 63;
        typedef decltype(__builtin_shufflevector(v, v, 0, 1, 2, 3)) quarter;
        typedef __attribute__((address_space(3))) quarter lds_quarter;
        lds_quarter *to = (lds_quarter *)(lds + (j * 32 + (lane & 31)) * kPitch + (i * 32 + (lane >> 5) * 4) * 4);
        to[0] = __builtin_shufflevector(v, v, 0, 1, 2, 3);
        to[2] = __builtin_shufflevector(v, v, 4, 5, 6, 7);
        to[4] = __builtin_shufflevector(v, v, 8, 9, 10, 11);
        to[6] = __builtin_shufflevector(v, v, 12, 13, 14, 15);
    }
    template <class Value>
    static __device__ __forceinline__ void take(const lds_char *lds, int row, int half, Value (&v)[8])
    {
        typedef Value quarter __attribute__((ext_vector_type(4)));
        const __attribute__((address_space(3))) quarter *from =
            (const __attribute__((address_space(3))) quarter *)(lds + row * kPitch + (((int)threadIdx.x & (kLanes - 1)) * 8 + half * (kCols / 2)) * 4);
        const quarter a = from[0], b = from[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    }
};
// Every row of the tile, a wave's quarter: column c of the tile's (kPair: of its half) and seven more of every row are a lane's.  fetch(row, c) asks for what else a row needs, kAhead
// rows at once before any of them is stored (loads are not moved over stores, and one at a time each waits for memory); use(row, c, v, u, fetched).
template <int kP, int kQ, bool kPair, class Product, class Fetch, class Use>
__device__ __forceinline__ void tile_results(const Product &t, lds_char *lds, Fetch fetch, Use use)
{
    typedef tile_out<kP, kQ, kPair> out;
    typedef decltype(t.acc[0][0][0] + t.acc[0][0][0]) value;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    lds_char *mine = lds + wave * out::kBytes;
    const int c = (wave & 1) * (kPair ? kP / 4 : kP / 2) + (lane & (out::kLanes - 1)) * 8;
    constexpr int kJ = out::kRows / 32, kTimes = out::kRows / out::kAtOnce, kAhead = kTimes < 8 ? kTimes : 8;
#pragma unroll
    for (int j = 0; j < Product::kNQ; j += kJ) {
#pragma unroll
        for (int i = 0; i < Product::kNP; ++i)
#pragma unroll
            for (int n = 0; n < kJ; ++n) out::put(mine, i, n, t.acc[i][j + n]);
        wave_order();
        const int row0 = (wave >> 1) * (kQ / 2) + j * 32;
#pragma unroll 1
        for (int n = 0; n < kTimes; n += kAhead) {
            decltype(fetch(0, 0)) more[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) more[i] = fetch(row0 + (n + i) * out::kAtOnce + lane / out::kLanes, c);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int row = (n + i) * out::kAtOnce + lane / out::kLanes;
                value v[8], u[8];
                out::take(mine, row, 0, v);
                if constexpr (kPair) out::take(mine, row, 1, u);
                use(row0 + row, c, v, kPair ? u : v, more[i]);
            }
        }
        wave_order();
    }
}

// The same where results are only rounded to bf16: rounded before they go through LDS, half the bytes both ways.  use(row, c, eight values).
template <int kP, int kQ>
struct tile_out_bf16 {
    static constexpr int kCols = kP / 2, kPitch = kCols * 2 + 16, kBytes = 32 * kPitch, kLanes = kCols / 8, kAtOnce = 64 / kLanes;
};
template <int kP, int kQ, class Product, class Use>
__device__ __forceinline__ void tile_results_bf16(const Product &t, lds_char *lds, Use use)
{
    typedef tile_out_bf16<kP, kQ> out;
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) bf16x4 lds_four;
    typedef const __attribute__((address_space(3))) u32x4 lds_eight;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    lds_char *mine = lds + wave * out::kBytes;
#pragma unroll
    for (int j = 0; j < Product::kNQ; ++j) {
#pragma unroll
        for (int i = 0; i < Product::kNP; ++i) {
            lds_char *to = mine + (lane & 31) * out::kPitch + (i * 32 + (lane >> 5) * 4) * 2;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (__bf16)t.acc[i][j][q * 4 + e];
                *(lds_four *)(to + q * 16) = v;
            }
        }
        wave_order();
#pragma unroll
        for (int n = 0; n < 32 / out::kAtOnce; ++n) {
            const int row = n * out::kAtOnce + lane / out::kLanes, c = (lane & (out::kLanes - 1)) * 8;
            use((wave >> 1) * (kQ / 2) + j * 32 + row, (wave & 1) * (kP / 2) + c, *(lds_eight *)(mine + row * out::kPitch + c * 2));
        }
        wave_order();
    }
}

// A product's kernels.  Op has: args (with g, p_tiles, K and parts, memory for kRound tiles' sums or null); kP, kQ, kTrP, kInt8; kPair: half of a wave's columns belong to
// the other half; feeds(): what is loaded; emit(): what becomes of eight columns of a row, with what columns() gives for the columns, rows() for the row (kRowValues: two
// values at most, which wait in LDS) and fetch() for both.
template <class Op>
struct tile_op : Op {
    typedef tile_product<Op::kP, Op::kQ, Op::kTrP, false, Op::kInt8> product;
    typedef tile_out<Op::kP, Op::kQ, Op::kPair> out;
    typedef decltype(typename product::kind::acc{}[0] + 0) value;
    // Workgroups that run at a time: LDS holds one of the two larger tiles a CU, two of 128 x 64 (with room for three steps each: with two, three
    // workgroups a CU, calls of a few tiles take 2 to 12 % longer, those of many up to 2 % less; with four, one a CU, they are 5 % slower than with three; 256 x 128 gains nothing from a third).
    static constexpr uint32_t kRound = Op::kP * Op::kQ > 128 * 128 ? 256 : 512;
    static constexpr int kLds = product::kLds > kTileWaves * out::kBytes ? product::kLds : kTileWaves * out::kBytes;
    static constexpr int kRowsAt = kLds, kAllLds = kLds + (Op::kRowValues ? 8 * Op::kQ : 0);           // a row's values behind the stages
    static constexpr int kColumns = Op::kPair ? Op::kP / 2 : Op::kP, kJoinRows = kTileThreads * 8 / kColumns;         // rows that a workgroup of k_join takes
    static __host__ __device__ __forceinline__ int steps(const typename Op::args &a) { return (a.K + (Op::kInt8 ? 127 : 63)) / (Op::kInt8 ? 128 : 64); }
    // Eight sums of a part, at a row and a column of a tile of kP columns.
    typedef value eight __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ eight *place(const typename Op::args &a, uint32_t slot, int row, int column) { return (eight *)((value *)a.parts + ((int64_t)slot * Op::kQ + row) * Op::kP + column); }
    // Column of a tile in a part, from a column that emit() has: waves' columns are kP / 2 each, the two halves of a pair behind one another.
    static __device__ __forceinline__ int column_of(int column, int half) { return Op::kPair ? column / (Op::kP / 4) * (Op::kP / 2) + column % (Op::kP / 4) + half * (Op::kP / 4) : column; }
};
template <class Op>
__global__ __launch_bounds__(kTileThreads, Op::kP * Op::kQ > 128 * 128 ? 1 : 2) void k_tiles(typename Op::args a)
{
    typedef tile_op<Op> op;
    typedef typename op::product product;
    __shared__ __attribute__((aligned(1024))) char lds[op::kAllLds];
    tile_runs<Op::kQ> runs;
    runs.count(a.g);
    const int steps = op::steps(a);
    const tile_split split = split_tiles(runs.total * (uint32_t)a.p_tiles, op::kRound, (uint32_t)steps, a.parts != nullptr);
    tile_unit u;
    tile_at at;
    if (!unit_of_workgroup(split, u) || !runs.find(a.g, (uint32_t)a.p_tiles, u.tile, at)) return;
    tile_feed<Op::kP, Op::kTrP, Op::kInt8> fp;
    tile_feed<Op::kQ, false, Op::kInt8> fq;
    Op::feeds(a, at, fp, fq);
    const bool part = u.tile >= split.whole && split.parts > 1;
    const int k0 = part ? (int)(u.part * (uint32_t)steps / split.parts) : 0, n = (part ? (int)((u.part + 1) * (uint32_t)steps / split.parts) : steps) - k0;
    if (part) {
        fp.part(k0, n);
        fq.part(k0, n);
    }
    f32x2 of_row = {};                               // (asked for before the stages' loads, kept until they are through)
    if constexpr (Op::kRowValues) if ((int)threadIdx.x < min(Op::kQ, at.rows) && !part) of_row = Op::rows(a, at.first + (int)threadIdx.x);
    product t;
    t.run(fp, fq, n, (lds_char *)lds);
    const uint32_t slot = u.part * split.rest + u.tile - split.whole;
    typedef typename op::value value;
    if (part) {
        tile_results<Op::kP, Op::kQ, Op::kPair>(t, (lds_char *)lds, [](int, int) { return 0; }, [&](int row, int column, const value (&v)[8], const value (&w)[8], int) {
            *op::place(a, slot, row, op::column_of(column, 0)) = typename op::eight{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
            if constexpr (Op::kPair) *op::place(a, slot, row, op::column_of(column, 1)) = typename op::eight{w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
        });
        return;
    }
    f32x2 *rows = (f32x2 *)(lds + op::kRowsAt);
    if constexpr (Op::kRowValues) {
        if ((int)threadIdx.x < Op::kQ) rows[threadIdx.x] = of_row;
        mw_lds_barrier();
    }
    const auto columns = Op::columns(a, at, (int)(threadIdx.x >> 6 & 1) * (op::kColumns / 2) + (int)(threadIdx.x & (op::out::kLanes - 1)) * 8);
    tile_results<Op::kP, Op::kQ, Op::kPair>(
        t, (lds_char *)lds, [&](int row, int column) { return Op::fetch(a, at, row, column); },
        [&](int row, int column, const value (&v)[8], const value (&w)[8], const decltype(Op::fetch(a, at, 0, 0)) &more) {
            Op::emit(a, at, row, column, v, w, columns, Op::kRowValues ? rows[row] : f32x2{}, more);
        });
}
// The parts' sums in their order.  grid: (kJoinRows rows of a tile, tiles in parts at most)
template <class Op>
__global__ __launch_bounds__(kTileThreads) void k_join(typename Op::args a)
{
    typedef tile_op<Op> op;
    tile_runs<Op::kQ> runs;
    runs.count(a.g);
    const tile_split split = split_tiles(runs.total * (uint32_t)a.p_tiles, op::kRound, (uint32_t)op::steps(a), true);
    tile_at at;
    if (split.parts == 1 || blockIdx.y >= split.rest || !runs.find(a.g, (uint32_t)a.p_tiles, split.whole + blockIdx.y, at)) return;
    const int row = (int)blockIdx.x * op::kJoinRows + (int)threadIdx.x / (op::kColumns / 8), column = (int)threadIdx.x % (op::kColumns / 8) * 8;
    if ((int)blockIdx.x * op::kJoinRows >= at.rows) return;
    typename op::eight v = {}, w = {};
#pragma unroll 4
    for (uint32_t n = 0; n < split.parts; ++n) {
        v += *op::place(a, n * split.rest + blockIdx.y, row, op::column_of(column, 0));
        if constexpr (Op::kPair) w += *op::place(a, n * split.rest + blockIdx.y, row, op::column_of(column, 1));
    }
    typename op::value x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { x[e] = v[e]; y[e] = w[e]; }
    f32x2 of_row = {};
    if constexpr (Op::kRowValues) if (row < at.rows) of_row = Op::rows(a, at.first + row);
    Op::emit(a, at, row, column, x, y, Op::columns(a, at, column), of_row, Op::fetch(a, at, row, column));
}
static inline int64_t most_tiles(int64_t n_rows, int64_t n, int rows_a_tile) { return n_rows / rows_a_tile + (n < n_rows ? n : n_rows); }
// Whether there may be parts is settled by the host, from the fewest tiles that so many rows are (after whole rounds the rest can be any number); how many there are, on the device by the runs' lengths.
static inline bool may_have_parts(int64_t n_rows, int64_t n, int rows_a_tile, int64_t column_tiles, int64_t steps)
{
    const int64_t rows_tiles = (n_rows + rows_a_tile - 1) / rows_a_tile, runs = n < n_rows ? n : n_rows, fewest = (rows_tiles > runs ? rows_tiles : runs) * column_tiles;
    return parts_pay((uint32_t)(fewest < kUnits ? fewest : kUnits / 2), (uint32_t)steps);
}
template <class Op>
int32_t launch_tiles(typename Op::args a, int columns, hipStream_t s)
{
    typedef tile_op<Op> op;
    a.p_tiles = (columns + (Op::kPair ? Op::kP / 2 : Op::kP) - 1) / (Op::kPair ? Op::kP / 2 : Op::kP);
    if (!may_have_parts(a.g.n_rows, a.g.n, Op::kQ, a.p_tiles, op::steps(a))) a.parts = nullptr;
    const int64_t tiles = most_tiles(a.g.n_rows, a.g.n, Op::kQ) * a.p_tiles, round = a.parts ? op::kRound : 0;
    if (tiles > 0x7ff00000LL) return MW_ERR_UNSUPPORTED;
    // T tiles are at most T - rest + kRound units, eights of them
    hipLaunchKernelGGL((k_tiles<Op>), grid_of((uint32_t)((tiles + round + 15) / 8 * 8)), dim3(kTileThreads), 0, s, a);
    MW_HIP_CHECK(hipGetLastError());
    if (a.parts) {
        hipLaunchKernelGGL((k_join<Op>), dim3(Op::kQ / op::kJoinRows, (uint32_t)(tiles < kUnits ? tiles : kUnits)), dim3(kTileThreads), 0, s, a);
        MW_HIP_CHECK(hipGetLastError());
    }
    return MW_OK;
}

__device__ __forceinline__ float tile_sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }
// kStreaming: past the caches.
template <bool kStreaming = false>
__device__ __forceinline__ void store_bf16(uint16_t *to, const float (&v)[8])
{
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)v[i];
    if constexpr (kStreaming) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, o), (u32x4 *)to);
    else *(bf16x8 *)to = o;
}

}  // namespace
#endif  // MW_TILE_H_
