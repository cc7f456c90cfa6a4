// Dense 16-bit product on the matrix cores, D = A B^T with fp32 accumulators:
// A [M][K] and B [N][K] row-major, or both given transposed (A [K][M] and
// B [K][N], the sum running over rows), and an epilogue that consumes a
// workgroup's D tile in registers.
//
//  * K may be split over workgroups (each split's D is an fp32 sum of its own).
//  * A workgroup of WM x WN waves owns a (WM * AM * 32) x (WN * AN * 32) tile;
//    each wave accumulates AM x AN blocks of v_mfma_f32_32x32x16 (rows from A,
//    columns from B).
//  * K is walked in chunks of 64.  Both operands reach LDS by direct-to-LDS
//    loads (no registers, no staging arithmetic) into one of two stages: chunk
//    c + 1 lands while chunk c is multiplied, one barrier a chunk.
//  * LDS row r (128 bytes, eight 16-byte slots) holds its values 8 s .. in slot
//    s ^ (r / 2 & 7): two rows fill the 256 bytes that LDS delivers a cycle, and
//    the sixteen rows of a fragment read then meet no bank twice (counters: no
//    conflict).  The direct-to-LDS destination
//    is fixed (lane l writes base + 16 l), so the permutation is on the source
//    address; it is the same for every row of a thread.
//  * Transposed operands keep their layout in LDS: a chunk is 64 rows of a
//    tile's columns, and the transposing LDS read gathers a lane's eight values
//    of K from eight rows, four at a time.  Row r's slots are moved by 4 (r & 3),
//    so that the four rows of a read lie in different bank groups.
//  * Measured, 256 x 256 tiles, bf16: 16384 x 4096 x 4096 0.41 ms, 1.33 PFLOP/s,
//    where a library's 8192^3 reaches 1.36; transposed operands 0.42 to 0.46 ms.
//    The matrix cores bound it, at the clock that the power leaves them.
//  * Rows past M or N are read from the last row (their results are dropped);
//    slots past K are read from a block of zeros.
#pragma once

#include <algorithm>
#include <type_traits>

#include "aq_device.h"

namespace aq {

struct GemmOperands {
    const uint16_t* A;
    const uint16_t* B;
    int64_t lda, ldb;      // row pitches in elements (multiples of 8, at most kMaxPitch; a transposed operand's
                           // K rows in all at most 4 GiB)
    int M, N, K;           // K a multiple of 8 (transposed operands: any K, rows of whole 16-byte groups)
    const uint8_t* zero;   // 16 zero bytes
    int tiles_m, tiles_n;
    int rows_fast;         // tiles of a band that share their B rows (see gemm_tile)
    int cps;               // K chunks a split
};

constexpr int kGemmChunk = 64;
// a tile's 256 rows, of fp32 sums too, stay below byte offset kOutOfRange
constexpr int64_t kMaxPitch = 1 << 21;
// tiles of 128 x 128 a launch may hold (fewer than 2^32 threads, K splits included)
constexpr int64_t kMaxTiles = 1 << 22;

template <int DT>
__device__ __forceinline__ floatx16 mfma_gemm(const u32x4& a, const u32x4& b, const floatx16& c) {
    if constexpr (DT == AQ_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0,
                                                      0, 0);
}

// Transposing LDS reads.  Within each sixteen lanes, lane 4 j + q names four
// neighbouring values of row j (columns 4 q ..), and lane l receives column l's
// values of the rows 0..3.  An operand comes from two of them, of rows 0..3 and
// 4..7 of its eight: eight values of one column.  Rows lie HB bytes apart in B's
// part of the stage (the first two operands) and HA in A's, step OFF 16 rows on.
// One block with its own wait: the compiler would hold its own reads of this
// kind until every load into LDS has landed, those of later chunks too.
template <int OFF, int HA, int HB>
__device__ __forceinline__ void lds_read_tr(const uint32_t (&a)[4], u32x4 (&o)[4]) {
    uint64_t r[8];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %2, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%14\n\t"
                 "ds_read_b64_tr_b16 %5, %10 offset:%15\n\t"
                 "ds_read_b64_tr_b16 %6, %11 offset:%14\n\t"
                 "ds_read_b64_tr_b16 %7, %11 offset:%15\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "n"(16 * OFF * HB), "n"((16 * OFF + 4) * HB),
                   "n"(16 * OFF * HA), "n"((16 * OFF + 4) * HA)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i)
        o[i] = u32x4{(uint32_t)r[2 * i], (uint32_t)(r[2 * i] >> 32), (uint32_t)r[2 * i + 1], (uint32_t)(r[2 * i + 1] >> 32)};
}
template <int OFF, int HA, int HB>
__device__ __forceinline__ void lds_read_tr(const uint32_t (&a)[6], u32x4 (&o)[6]) {
    uint64_t r[12];
    asm volatile("ds_read_b64_tr_b16 %0, %12 offset:%18\n\t"
                 "ds_read_b64_tr_b16 %1, %12 offset:%19\n\t"
                 "ds_read_b64_tr_b16 %2, %13 offset:%18\n\t"
                 "ds_read_b64_tr_b16 %3, %13 offset:%19\n\t"
                 "ds_read_b64_tr_b16 %4, %14 offset:%20\n\t"
                 "ds_read_b64_tr_b16 %5, %14 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %6, %15 offset:%20\n\t"
                 "ds_read_b64_tr_b16 %7, %15 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %8, %16 offset:%20\n\t"
                 "ds_read_b64_tr_b16 %9, %16 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %10, %17 offset:%20\n\t"
                 "ds_read_b64_tr_b16 %11, %17 offset:%21\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]),
                   "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "n"(16 * OFF * HB),
                   "n"((16 * OFF + 4) * HB), "n"(16 * OFF * HA), "n"((16 * OFF + 4) * HA)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 6; ++i)
        o[i] = u32x4{(uint32_t)r[2 * i], (uint32_t)(r[2 * i] >> 32), (uint32_t)r[2 * i + 1], (uint32_t)(r[2 * i + 1] >> 32)};
}

// Row of D that accumulator register r of a lane holds within its 32 x 32 block.
__device__ __forceinline__ int gemm_row(int r, int hi) { return 8 * (r >> 2) + 4 * hi + (r & 3); }

template <int WM, int WN, int AM, int AN>
struct GemmTile {
    static constexpr int kThreads = WM * WN * 64;
    static constexpr int BM = WM * AM * 32, BN = WN * AN * 32;
    static constexpr int kStage = (BM + BN) * kGemmChunk * 2;   // bytes
    static constexpr int kLds = 2 * kStage;
    static constexpr int LA = BM * 8 / kThreads, LB = BN * 8 / kThreads;   // 16-byte loads a thread and chunk
    static_assert(BM * 8 % kThreads == 0 && BN * 8 % kThreads == 0, "whole loads");
    static_assert(kThreads % 64 == 0 && kThreads / 8 % 16 == 0, "one slot permutation a thread");
};

// Tile of this workgroup: consecutive workgroups go to different XCDs, so each
// XCD takes a contiguous run of tiles; a run walks bands of `rows_fast` tiles
// along M, column by column, so that its L2 serves both operands.
__device__ __forceinline__ void gemm_tile(const GemmOperands& g, int& tm, int& tn, int& z) {
    const int nwg = (int)gridDim.x, h = (int)blockIdx.x;
    const int xcd = h & 7, j = h >> 3;
    const int per = nwg >> 3, rem = nwg & 7;
    int w = xcd * per + min(xcd, rem) + j;
    z = w / (g.tiles_m * g.tiles_n);
    w -= z * g.tiles_m * g.tiles_n;
    const int band = w / (g.rows_fast * g.tiles_n);
    const int m0 = band * g.rows_fast;
    const int rows = min(g.rows_fast, g.tiles_m - m0);
    const int in = w - band * g.rows_fast * g.tiles_n;
    tn = in / rows;
    tm = m0 + in - tn * rows;
}

// Accumulators of D's tile at (m0, n0) over K chunks [c_beg, c_end).
template <int DT, int WM, int WN, int AM, int AN, bool TR>
__device__ __forceinline__ void gemm_mainloop(const GemmOperands& g, int m0, int n0, int c_beg, int c_end, uint8_t* lds,
                                              floatx16 (&acc)[AM][AN]) {
    using T = GemmTile<WM, WN, AM, AN>;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave - wm * WN;
    const int l32 = lane & 31, hi = lane >> 5;

    // One load a thread: 16 bytes of a row; whole chunks go through buffer loads (the row's offset in a
    // register, the chunk's in a scalar: no address arithmetic), the last part of a chunk through addresses
    // that point past K's end at the zero block.
    const uint16_t* ta = g.A + (TR ? (int64_t)m0 : (int64_t)m0 * g.lda);
    const uint16_t* tb = g.B + (TR ? (int64_t)n0 : (int64_t)n0 * g.ldb);
    const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(ta, 0xFFFFFFFFu), rb = buffer_rsrc(tb, 0xFFFFFFFFu);
    // plain: rows tid / 8 + j * threads / 8 of the tile, eight slots a row along K;
    // transposed: rows of K, tid / (slots a row) + j * ..., slots along M or N
    constexpr int kRows = T::kThreads / 8;
    constexpr int SA = T::BM / 8, SB = T::BN / 8;                // transposed: slots a row
    const int r0 = tid >> 3;
    const int slot = (tid & 7) ^ ((r0 >> 1) & 7);
    const int ka = tid / SA, kb = tid / SB;                      // transposed: first row of K
    uint32_t oa[T::LA], ob[T::LB];
    if constexpr (TR) {
        const int ca = min(8 * ((tid % SA) ^ ((ka & 3) << 2)), (g.M - 1 - m0) & ~7);
        const int cb = min(8 * ((tid % SB) ^ ((kb & 3) << 2)), (g.N - 1 - n0) & ~7);
#pragma unroll
        for (int j = 0; j < T::LA; ++j) oa[j] = (uint32_t)((ka + j * (T::kThreads / SA)) * (int)g.lda + ca) * 2u;
#pragma unroll
        for (int j = 0; j < T::LB; ++j) ob[j] = (uint32_t)((kb + j * (T::kThreads / SB)) * (int)g.ldb + cb) * 2u;
    } else {
        const int ma = min(T::BM, g.M - m0) - 1, mb = min(T::BN, g.N - n0) - 1;
#pragma unroll
        for (int j = 0; j < T::LA; ++j) oa[j] = (uint32_t)(min(r0 + j * kRows, ma) * (int)g.lda + 8 * slot) * 2u;
#pragma unroll
        for (int j = 0; j < T::LB; ++j) ob[j] = (uint32_t)(min(r0 + j * kRows, mb) * (int)g.ldb + 8 * slot) * 2u;
    }
    // bytes from one chunk to the next
    const uint32_t sa = TR ? (uint32_t)g.lda * (kGemmChunk * 2u) : kGemmChunk * 2u;
    const uint32_t sb = TR ? (uint32_t)g.ldb * (kGemmChunk * 2u) : kGemmChunk * 2u;
    auto issue_whole = [&](int i, int chunk, uint8_t* st) {      // load i of LA + LB of a whole chunk
        const uint32_t off = i < T::LA ? oa[i < T::LA ? i : 0] : ob[i < T::LA ? 0 : i - T::LA];
        lds_dma16(i < T::LA ? ra : rb, off, (uint32_t)chunk * (i < T::LA ? sa : sb),
                  st + (i * T::kThreads + wave * 64) * 16);
    };
    auto issue_one = [&](int i, int chunk, uint8_t* st) {
        if (chunk * kGemmChunk + kGemmChunk <= g.K) {
            issue_whole(i, chunk, st);
        } else {
            const uint32_t off = i < T::LA ? oa[i < T::LA ? i : 0] : ob[i < T::LA ? 0 : i - T::LA];
            const uint8_t* p = reinterpret_cast<const uint8_t*>(i < T::LA ? ta : tb) +
                               (int64_t)chunk * (i < T::LA ? sa : sb) + off;
            const int k = TR ? (i < T::LA ? ka + i * (T::kThreads / SA) : kb + (i - T::LA) * (T::kThreads / SB)) : 8 * slot;
            lds_dma16(chunk * kGemmChunk + k < g.K ? p : g.zero, st + (i * T::kThreads + wave * 64) * 16);
        }
    };
    auto issue = [&](int chunk, uint8_t* st) {
#pragma unroll
        for (int i = 0; i < T::LA + T::LB; ++i) issue_one(i, chunk, st);
    };
#pragma unroll
    for (int a = 0; a < AM; ++a)
#pragma unroll
        for (int b = 0; b < AN; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;

    const uint32_t arow = (uint32_t)(wm * AM * 32 + l32) * 128u;
    const uint32_t brow = (uint32_t)(T::BM + wn * AN * 32 + l32) * 128u;
    // operands of step s (16 values of K) of a stage: one by one, or transposed all at once
    auto operand = [&](const uint8_t* st, int s, int i) {
        const uint32_t off = (uint32_t)(((2 * s + hi) ^ ((l32 >> 1) & 7)) * 16);
        return *reinterpret_cast<const u32x4*>(st + (i < AN ? brow + i * 4096 : arow + (i - AN) * 4096) + off);
    };
    uint32_t tr[AN + AM];      // this lane's place in rows 8 * hi + (lane & 15) / 4 of step 0
    if constexpr (TR) {
        const int r = (lane >> 2) & 3;
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
#pragma unroll
        for (int i = 0; i < AN + AM; ++i) {
            const int blk = i < AN ? wn * AN + i : wm * AM + i - AN;           // block of 32 columns
            const int sl = 4 * (blk ^ r) + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
            tr[i] = base + (uint32_t)((i < AN ? T::BM * 128 : 0) + (8 * hi + r) * (i < AN ? T::BN : T::BM) * 2 + sl * 16 +
                                      (lane & 1) * 8);
        }
    }
    auto operands_tr = [&](uint32_t stage, auto s, u32x4 (&f)[AN + AM]) {
        uint32_t at[AN + AM];
#pragma unroll
        for (int i = 0; i < AN + AM; ++i) at[i] = tr[i] + stage;
        lds_read_tr<decltype(s)::value, T::BM * 2, T::BN * 2>(at, f);
    };
    if (c_beg >= c_end) return;
    // Step s + 1's operands are read between step s's products.  A chunk's last step multiplies after the
    // barrier that hands over its stage, so that the next chunk's first operands and the loads of the
    // chunk after it are on their way under those products.
    u32x4 f[2][AN + AM];
    constexpr int kOps = AN + AM, kProducts = AM * AN, kLoads = T::LA + T::LB;
    issue(c_beg, lds);
    wait_vmcnt<0>();
    lds_barrier();
    if (c_beg + 1 < c_end) issue(c_beg + 1, lds + T::kStage);
    if constexpr (TR) {
        operands_tr(0, std::integral_constant<int, 0>{}, f[0]);
    } else {
#pragma unroll
        for (int i = 0; i < kOps; ++i) f[0][i] = operand(lds, 0, i);
    }
    // The reads are early in a step, so that the wait for them finds them done; transposing ones, which wait for
    // themselves, stand behind a quarter of the products (the other wave of the SIMD multiplies meanwhile).
    auto step = [&](uint32_t from, auto sc, auto&& load) {
        constexpr int s = decltype(sc)::value;
#pragma unroll
        for (int i = 0; i < kProducts; ++i) {
            if constexpr (TR) {
                if (i == kProducts / 4) operands_tr(from, std::integral_constant<int, (s + 1) & 3>{}, f[(s + 1) & 1]);
            } else {
#pragma unroll
                for (int q = 2 * i; q < min(2 * i + 2, kOps); ++q) f[(s + 1) & 1][q] = operand(lds + from, (s + 1) & 3, q);
            }
            load(i);
            acc[i / AN][i % AN] = mfma_gemm<DT>(f[s & 1][AN + i / AN], f[s & 1][i % AN], acc[i / AN][i % AN]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto none = [](int) {};
    auto three = [&](uint32_t st) {
        step(st, std::integral_constant<int, 0>{}, none);
        step(st, std::integral_constant<int, 1>{}, none);
        step(st, std::integral_constant<int, 2>{}, none);
    };
    int c = c_beg;
    for (; c + 2 < c_end && (c + 3) * kGemmChunk <= g.K; ++c) {       // the chunk loaded is a whole one
        const uint32_t st = (uint32_t)((c - c_beg) & 1) * T::kStage, next = T::kStage - st;
        three(st);
        wait_vmcnt<0>();      // this wave's part of chunk c + 1 landed
        lds_barrier();        // everyone's; and every wave has read all of chunk c
        step(next, std::integral_constant<int, 3>{}, [&](int i) {
#pragma unroll
            for (int q = i * kLoads / kProducts; q < (i + 1) * kLoads / kProducts; ++q) issue_whole(q, c + 2, lds + st);
        });
    }
    for (; c < c_end; ++c) {                                         // the last two or three
        const uint32_t st = (uint32_t)((c - c_beg) & 1) * T::kStage, next = T::kStage - st;
        three(st);
        if (c + 1 < c_end) {
            wait_vmcnt<0>();
            lds_barrier();
            if (c + 2 < c_end) issue(c + 2, lds + st);
        }
        step(next, std::integral_constant<int, 3>{}, none);   // (the last chunk's reads of the other stage are not used)
    }
}

// Where a product's D goes: 16-bit results, or fp32 sums that later products
// of the same output add to.  With K split over workgroups every split keeps a
// sum of its own, and split_sum_kernel adds them.
enum StoreMode {
    STORE_OUT = 0,         // out = D, unscaled
    STORE_SUM = 1,         // sum = D
    STORE_ADD = 2,         // sum += D
    STORE_LAST = 3         // out = sum + D, unscaled
};

// The logits' gradient is stored in 16 bits, scaled so that an entry at a target, `peak`, lies at 32640 = 255 * 2^7,
// which fp16 and bf16 hold exactly, near the end of a binade: the entries that make most of a row's gradient, which
// share one rounding, then round with half the error of the worst scale (the peak with none).  For dW, and for both in
// bf16, whose exponents are fp32's, it is the largest such entry of the call.  fp16 holds 39 binades below it, and
// rows of far smaller weights would lose their small entries: for dX, whose rows stand apart, it is each token's own.
constexpr float kGradPeak = 32640.0f;
constexpr bool own_peaks(int dtype) { return dtype == AQ_F16; }       // dX's operand is scaled token by token
__device__ __forceinline__ bool peak_fits(float peak) { return peak > 0x1p-100f; }      // (a quotient below would overflow)
__device__ __forceinline__ float grad_scale(float peak) { return peak_fits(peak) ? kGradPeak / peak : 1.0f; }
__device__ __forceinline__ float grad_unscale(float peak) { return peak_fits(peak) ? peak / kGradPeak : 1.0f; }

template <int DT>
struct StoreArgs {
    uint16_t* out;         // [M] rows of pitch ldo
    float* sum;            // [split][M][N]
    int64_t ldo;           // at most kMaxPitch, as N is
    const float* peak;     // of a scaled gradient; null: D as it is
    const float* own;      // peaks of D's rows instead (where they have their own)
};

// OWN: D's rows have peaks of their own.
template <int DT, int MODE, bool OWN, int WM, int WN, int AM, int AN>
struct StoreEpilogue {
    StoreArgs<DT> s;

    // Branch-free buffer accesses at offsets from the tile's corner; positions past D's edge get an offset past
    // the buffer.
    __device__ void operator()(const floatx16 (&acc)[AM][AN], int, int z, int m0, int n0, int M, int N, uint8_t*) const {
        constexpr bool kOut = MODE == STORE_OUT || MODE == STORE_LAST, kOld = MODE == STORE_ADD || MODE == STORE_LAST;
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int wm = wave / WN, wn = wave - wm * WN, l32 = lane & 31, hi = lane >> 5;
        const float f = kOut && !OWN && s.peak ? grad_unscale(*s.peak) : 1.0f;
        const __amdgpu_buffer_rsrc_t ro = buffer_rsrc(s.out + (int64_t)m0 * s.ldo + n0, kOutOfRange);
        const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(s.sum + ((int64_t)z * M + m0) * N + n0, kOutOfRange);
#pragma unroll
        for (int a = 0; a < AM; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int m = (wm * AM + a) * 32 + gemm_row(r, hi);
                const float fm = kOut && OWN ? grad_unscale(s.own[min(m0 + m, M - 1)]) : f;
#pragma unroll
                for (int b = 0; b < AN; ++b) {
                    const int n = (wn * AN + b) * 32 + l32;
                    const bool in = m0 + m < M && n0 + n < N;
                    const uint32_t os = in ? (uint32_t)(m * N + n) * 4u : kOutOfRange;
                    float v = acc[a][b][r];
                    if (kOld) v += __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, os, 0, 0));
                    if (kOut) {
                        const uint32_t oo = in ? (uint32_t)(m * (int)s.ldo + n) * 2u : kOutOfRange;
                        __builtin_amdgcn_raw_buffer_store_b16(f32_to_tile<DT>(v * fm), ro, oo, 0, 0);
                    } else {
                        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), rs, os, 0, 0);
                    }
                }
            }
    }
};

template <int DT, int WM, int WN, int AM, int AN, bool TR, class Epi>
__global__ void __launch_bounds__(WM* WN * 64, WM* WN == 8 ? 1 : 2) gemm_kernel(GemmOperands g, Epi epi) {
    using T = GemmTile<WM, WN, AM, AN>;
    extern __shared__ __attribute__((aligned(16))) uint8_t gemm_lds[];
    int tm, tn, z;
    gemm_tile(g, tm, tn, z);
    const int chunks = (g.K + kGemmChunk - 1) / kGemmChunk;
    floatx16 acc[AM][AN];
    gemm_mainloop<DT, WM, WN, AM, AN, TR>(g, tm * T::BM, tn * T::BN, z * g.cps, min(chunks, (z + 1) * g.cps), gemm_lds, acc);
    epi(acc, tm, z, tm * T::BM, tn * T::BN, g.M, g.N, gemm_lds);
}

// Tile and K split of one product.
struct GemmPlan {
    bool big;              // 256 x 256 tiles of eight waves, else 128 x 128 of four
    int splits, cps;       // splits (every one owns a chunk), chunks a split
};

// Shortest by a model of the calls: rounds of 256 big or 512 small tiles (one
// or two a compute unit), a tile's fixed time and its time a chunk, and the
// splits' sums.  `cap`: bytes there are for them (0: no splits).
inline GemmPlan gemm_plan(int64_t M, int64_t N, int64_t K, size_t cap) {
    const int chunks = (int)((K + kGemmChunk - 1) / kGemmChunk);
    GemmPlan best{true, 1, chunks};
    double best_us = 1e30;
    for (int big = 1; big >= 0; --big) {
        const int64_t side = big ? 256 : 128, slots = big ? 256 : 512;
        const int64_t tiles = (M + side - 1) / side * ((N + side - 1) / side);
        const double fixed = big ? 12.0 : 7.0;
        for (int s = 1; s <= std::min(chunks, 64); ++s) {
            if (s > 1 && (tiles * (s - 1) >= slots || (size_t)s * M * N * 4 > cap)) break;
            const int cps = (chunks + s - 1) / s;
            if ((chunks + cps - 1) / cps != s) continue;
            const int64_t rounds = (tiles * s + slots - 1) / slots;
            const double chunk = big ? 1.6 : tiles * s <= 256 ? 0.65 : 1.3;
            const double us = rounds * (fixed + chunk * cps) + (s > 1 ? 4.0 + 1e-6 * M * N * s : 0.0);
            if (us < best_us) {
                best_us = us;
                best = GemmPlan{big != 0, s, cps};
            }
        }
    }
    return best;
}

// Bytes of the split sums that calls of up to max_rows rows plan within `cap`.  Fewer rows of the same tiles never
// split less (only the sums' time grows with the rows), so each step of 128 rows is bounded by its first row's splits.
inline size_t gemm_split_bytes(int64_t max_rows, int64_t N, int64_t K, size_t cap) {
    size_t need = 0;
    for (int64_t lo = 1; lo <= max_rows && lo <= 128 * 512; lo += 128) {
        const GemmPlan p = gemm_plan(lo, N, K, cap);
        if (p.splits > 1) need = std::max(need, (size_t)p.splits * std::min(lo + 127, max_rows) * N * 4);
    }
    return std::min(need, cap);
}

template <int DT, int WM, int WN, int AM, int AN, bool TR, class Epi>
hipError_t launch_gemm(GemmOperands g, const GemmPlan& p, const Epi& epi, hipStream_t st) {
    using T = GemmTile<WM, WN, AM, AN>;
    g.tiles_m = (g.M + T::BM - 1) / T::BM;
    g.tiles_n = (g.N + T::BN - 1) / T::BN;
    g.rows_fast = std::min(8, g.tiles_m);
    g.cps = p.cps;
    auto kern = gemm_kernel<DT, WM, WN, AM, AN, TR, Epi>;
    const hipError_t e = ensure_dynamic_lds((const void*)kern, T::kLds);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)((int64_t)g.tiles_m * g.tiles_n * p.splits), T::kThreads, T::kLds, st>>>(g, epi);
    return hipGetLastError();
}

template <int DT, bool TR, int MODE>
hipError_t launch_store_gemm(const GemmOperands& g, const GemmPlan& p, const StoreArgs<DT>& s, hipStream_t st) {
    constexpr bool kOwn = TR && own_peaks(DT);        // (transposed operands: dX)
    return p.big ? launch_gemm<DT, 2, 4, 4, 2, TR>(g, p, StoreEpilogue<DT, MODE, kOwn, 2, 4, 4, 2>{s}, st)
                 : launch_gemm<DT, 2, 2, 2, 2, TR>(g, p, StoreEpilogue<DT, MODE, kOwn, 2, 2, 2, 2>{s}, st);
}

// out[m][n] = unscaled (sum over the splits, in split order), four values a thread (N a multiple of 8).
// OWN: by the rows' own peaks.
template <int DT, bool OWN>
__global__ void __launch_bounds__(256) split_sum_kernel(const float* sum, int splits, int64_t M, int N, uint16_t* out,
                                                        int64_t ldo, const float* peak, const float* own) {
    const float call = !OWN && peak ? grad_unscale(*peak) : 1.0f;
    const int64_t count = M * N;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < count; i += (int64_t)gridDim.x * 1024) {
        floatx4 v = *reinterpret_cast<const floatx4*>(sum + i);
#pragma unroll 8
        for (int z = 1; z < splits; ++z) v += *reinterpret_cast<const floatx4*>(sum + z * count + i);
        const int64_t m = i / N;
        const float f = OWN ? grad_unscale(own[m]) : call;
        *reinterpret_cast<uint2*>(out + m * ldo + (i - m * N)) =
            make_uint2(f32_to_tile<DT>(v[0] * f) | (uint32_t)f32_to_tile<DT>(v[1] * f) << 16,
                       f32_to_tile<DT>(v[2] * f) | (uint32_t)f32_to_tile<DT>(v[3] * f) << 16);
    }
}

template <int DT, bool OWN>
hipError_t launch_split_sum(const float* sum, int splits, int64_t M, int N, uint16_t* out, int64_t ldo,
                            const float* peak, const float* own, hipStream_t st) {
    const int64_t blocks = (M * N + 1023) / 1024;
    split_sum_kernel<DT, OWN><<<(unsigned)std::min<int64_t>(blocks, 8192), 256, 0, st>>>(sum, splits, M, N, out, ldo, peak, own);
    return hipGetLastError();
}

}  // namespace aq
