// Dense 16-bit product on the matrix cores, D = A B^T with fp32 accumulators:
// A [M][K] and B [N][K] row-major (both with K contiguous), and an epilogue
// that consumes a workgroup's D tile in registers.
//
//  * K may be split over workgroups (each split's D is an fp32 sum of its own).
//  * A workgroup of WM x WN waves owns a (WM * AM * 32) x (WN * AN * 32) tile;
//    each wave accumulates AM x AN blocks of v_mfma_f32_32x32x16 (rows from A,
//    columns from B).
//  * K is walked in chunks of 64.  Both operands reach LDS by direct-to-LDS
//    loads (no registers, no staging arithmetic) into one of two stages: chunk
//    c + 1 lands while chunk c is multiplied, one barrier a chunk.
//  * LDS row r (128 bytes, eight 16-byte slots) holds its 64 values with slot
//    s = chunk s ^ (r & 7), so the eight rows that a fragment read touches at a
//    time lie in eight different bank groups.  The direct-to-LDS destination
//    is fixed (lane l writes base + 16 l), so the permutation is on the source
//    address; it is the same for every row of a thread.
//  * Rows past M or N are read from the last row (their results are dropped);
//    slots past K are read from a block of zeros.
#pragma once

#include <algorithm>

#include "aq_device.h"

namespace aq {

struct GemmOperands {
    const uint16_t* A;
    const uint16_t* B;
    int64_t lda, ldb;      // row pitches in elements (multiples of 8, at most kMaxPitch)
    int M, N, K;           // K a multiple of 8
    const uint8_t* zero;   // 16 zero bytes
    int tiles_m, tiles_n;
    int rows_fast;         // tiles of a band that share their B rows (see gemm_tile)
    int cps;               // K chunks a split
};

constexpr int kGemmChunk = 64;
// a tile's 255 rows stay within 32-bit byte offsets
constexpr int64_t kMaxPitch = 1 << 22;

template <int DT>
__device__ __forceinline__ floatx16 mfma_gemm(const u32x4& a, const u32x4& b, const floatx16& c) {
    if constexpr (DT == AQ_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0,
                                                      0, 0);
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
template <int DT, int WM, int WN, int AM, int AN>
__device__ __forceinline__ void gemm_mainloop(const GemmOperands& g, int m0, int n0, int c_beg, int c_end, uint8_t* lds,
                                              floatx16 (&acc)[AM][AN]) {
    using T = GemmTile<WM, WN, AM, AN>;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave - wm * WN;
    const int l32 = lane & 31, hi = lane >> 5;

    // One load a thread: 16 bytes of row r0 + j * rows; whole chunks go through buffer loads (the row's
    // offset in a register, the chunk's in a scalar: no address arithmetic), the last part of a chunk
    // through addresses that point past K's end at the zero block.
    constexpr int kRows = T::kThreads / 8;
    const int r0 = tid >> 3;
    const int slot = (tid & 7) ^ ((r0 >> 1) & 7);
    const uint16_t* ta = g.A + (int64_t)m0 * g.lda;
    const uint16_t* tb = g.B + (int64_t)n0 * g.ldb;
    const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(ta, 0xFFFFFFFFu), rb = buffer_rsrc(tb, 0xFFFFFFFFu);
    const int ma = min(T::BM, g.M - m0) - 1, mb = min(T::BN, g.N - n0) - 1;
    uint32_t oa[T::LA], ob[T::LB];
#pragma unroll
    for (int j = 0; j < T::LA; ++j) oa[j] = (uint32_t)(min(r0 + j * kRows, ma) * (int)g.lda + 8 * slot) * 2u;
#pragma unroll
    for (int j = 0; j < T::LB; ++j) ob[j] = (uint32_t)(min(r0 + j * kRows, mb) * (int)g.ldb + 8 * slot) * 2u;
    auto issue_whole = [&](int i, int chunk, uint8_t* st) {      // load i of LA + LB of a whole chunk
        const uint32_t off = i < T::LA ? oa[i < T::LA ? i : 0] : ob[i < T::LA ? 0 : i - T::LA];
        lds_dma16(i < T::LA ? ra : rb, off, (uint32_t)chunk * (kGemmChunk * 2u), st + (i * T::kThreads + wave * 64) * 16);
    };
    auto issue_one = [&](int i, int chunk, uint8_t* st) {
        uint8_t* dst = st + (i * T::kThreads + wave * 64) * 16;
        const int k0 = chunk * kGemmChunk;
        const uint32_t off = i < T::LA ? oa[i < T::LA ? i : 0] : ob[i < T::LA ? 0 : i - T::LA];
        if (k0 + kGemmChunk <= g.K) {
            lds_dma16(i < T::LA ? ra : rb, off, (uint32_t)k0 * 2u, dst);
        } else {
            const uint8_t* p = reinterpret_cast<const uint8_t*>((i < T::LA ? ta : tb) + k0) + off;
            lds_dma16(k0 + 8 * slot < g.K ? p : g.zero, dst);
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
    // operand i of AN + AM of step s (16 values of K) of a stage
    auto operand = [&](const uint8_t* st, int s, int i) {
        const uint32_t off = (uint32_t)(((2 * s + hi) ^ ((l32 >> 1) & 7)) * 16);
        return *reinterpret_cast<const u32x4*>(st + (i < AN ? brow + i * 4096 : arow + (i - AN) * 4096) + off);
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
#pragma unroll
    for (int i = 0; i < kOps; ++i) f[0][i] = operand(lds, 0, i);
    // the reads are early in a step, so that the wait for them finds them done
    auto step = [&](const uint8_t* from, int s, auto&& load) {
#pragma unroll
        for (int i = 0; i < kProducts; ++i) {
#pragma unroll
            for (int q = 2 * i; q < min(2 * i + 2, kOps); ++q) f[(s + 1) & 1][q] = operand(from, (s + 1) & 3, q);
            load(i);
            acc[i / AN][i % AN] = mfma_gemm<DT>(f[s & 1][AN + i / AN], f[s & 1][i % AN], acc[i / AN][i % AN]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto none = [](int) {};
    int c = c_beg;
    for (; c + 2 < c_end && (c + 3) * kGemmChunk <= g.K; ++c) {       // the chunk loaded is a whole one
        uint8_t* st = lds + ((c - c_beg) & 1) * T::kStage;
        uint8_t* next = lds + ((c + 1 - c_beg) & 1) * T::kStage;
#pragma unroll
        for (int s = 0; s < 3; ++s) step(st, s, none);
        wait_vmcnt<0>();      // this wave's part of chunk c + 1 landed
        lds_barrier();        // everyone's; and every wave has read all of chunk c
        step(next, 3, [&](int i) {
#pragma unroll
            for (int q = i * kLoads / kProducts; q < (i + 1) * kLoads / kProducts; ++q) issue_whole(q, c + 2, st);
        });
    }
    for (; c < c_end; ++c) {                                         // the last two or three
        uint8_t* st = lds + ((c - c_beg) & 1) * T::kStage;
        uint8_t* next = lds + ((c + 1 - c_beg) & 1) * T::kStage;
#pragma unroll
        for (int s = 0; s < 3; ++s) step(st, s, none);
        if (c + 1 < c_end) {
            wait_vmcnt<0>();
            lds_barrier();
            if (c + 2 < c_end) issue(c + 2, st);
        }
        step(next, 3, none);  // (the last chunk's reads of the other stage are not used)
    }
}

// Where a product's D goes: 16-bit results, or fp32 sums that later products
// of the same output add to.  With K split over workgroups every split keeps a
// sum of its own, and split_sum_kernel adds them.
enum StoreMode {
    STORE_OUT = 0,         // out = D * scale
    STORE_SUM = 1,         // sum = D
    STORE_ADD = 2,         // sum += D
    STORE_LAST = 3         // out = (sum + D) * scale
};

template <int DT>
struct StoreArgs {
    uint16_t* out;         // [M] rows of pitch ldo
    float* sum;            // [split][M][N]
    int64_t ldo;           // at most kMaxPitch, as N is
    const float* scale;    // null: 1
};

template <int DT, int MODE, int WM, int WN, int AM, int AN>
struct StoreEpilogue {
    StoreArgs<DT> s;

    // Branch-free buffer accesses at offsets from the tile's corner; positions past D's edge get an offset past
    // the buffer.
    __device__ void operator()(const floatx16 (&acc)[AM][AN], int, int z, int m0, int n0, int M, int N, uint8_t*) const {
        constexpr bool kOut = MODE == STORE_OUT || MODE == STORE_LAST, kOld = MODE == STORE_ADD || MODE == STORE_LAST;
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int wm = wave / WN, wn = wave - wm * WN, l32 = lane & 31, hi = lane >> 5;
        const float f = kOut && s.scale ? *s.scale : 1.0f;
        const __amdgpu_buffer_rsrc_t ro = buffer_rsrc(s.out + (int64_t)m0 * s.ldo + n0, kOutOfRange);
        const __amdgpu_buffer_rsrc_t rs = buffer_rsrc(s.sum + ((int64_t)z * M + m0) * N + n0, kOutOfRange);
#pragma unroll
        for (int a = 0; a < AM; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int m = (wm * AM + a) * 32 + gemm_row(r, hi);
#pragma unroll
                for (int b = 0; b < AN; ++b) {
                    const int n = (wn * AN + b) * 32 + l32;
                    const bool in = m0 + m < M && n0 + n < N;
                    const uint32_t os = in ? (uint32_t)(m * N + n) * 4u : kOutOfRange;
                    float v = acc[a][b][r];
                    if (kOld) v += __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, os, 0, 0));
                    if (kOut) {
                        const uint32_t oo = in ? (uint32_t)(m * (int)s.ldo + n) * 2u : kOutOfRange;
                        __builtin_amdgcn_raw_buffer_store_b16(f32_to_tile<DT>(v * f), ro, oo, 0, 0);
                    } else {
                        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), rs, os, 0, 0);
                    }
                }
            }
    }
};

template <int DT, int WM, int WN, int AM, int AN, class Epi>
__global__ void __launch_bounds__(WM* WN * 64, WM* WN == 8 ? 1 : 2) gemm_kernel(GemmOperands g, Epi epi) {
    using T = GemmTile<WM, WN, AM, AN>;
    extern __shared__ __attribute__((aligned(16))) uint8_t gemm_lds[];
    int tm, tn, z;
    gemm_tile(g, tm, tn, z);
    const int chunks = (g.K + kGemmChunk - 1) / kGemmChunk;
    floatx16 acc[AM][AN];
    gemm_mainloop<DT, WM, WN, AM, AN>(g, tm * T::BM, tn * T::BN, z * g.cps, min(chunks, (z + 1) * g.cps), gemm_lds, acc);
    epi(acc, tm, z, tm * T::BM, tn * T::BN, g.M, g.N, gemm_lds);
}

// Tile and K split of one product.
struct GemmPlan {
    bool big;              // 256 x 256 tiles of eight waves, else 128 x 128 of four
    int splits, cps;       // splits (every one owns a chunk), chunks a split
};

// Shortest by a model of the calls: rounds of 256 big or 512 small tiles (one
// or two a compute unit), a tile's fixed time and its time a chunk, and the
// splits' sums.
inline GemmPlan gemm_plan(int64_t M, int64_t N, int64_t K, bool may_split) {
    const int chunks = (int)((K + kGemmChunk - 1) / kGemmChunk);
    GemmPlan best{true, 1, chunks};
    double best_us = 1e30;
    for (int big = 1; big >= 0; --big) {
        const int64_t side = big ? 256 : 128, slots = big ? 256 : 512;
        const int64_t tiles = (M + side - 1) / side * ((N + side - 1) / side);
        const double fixed = big ? 6.0 : 4.0, chunk = big ? 1.75 : 1.0;
        for (int s = 1; s <= (may_split ? std::min(chunks, 64) : 1); ++s) {
            if (s > 1 && tiles * (s - 1) >= slots) break;
            const int cps = (chunks + s - 1) / s;
            if ((chunks + cps - 1) / cps != s) continue;
            const int64_t rounds = (tiles * s + slots - 1) / slots;
            const double us = rounds * (fixed + chunk * cps) + (s > 1 ? 4.0 + 8e-6 * M * N * s / 4 : 0.0);
            if (us < best_us) {
                best_us = us;
                best = GemmPlan{big != 0, s, cps};
            }
        }
    }
    return best;
}

template <int DT, int WM, int WN, int AM, int AN, class Epi>
hipError_t launch_gemm(GemmOperands g, const GemmPlan& p, const Epi& epi, hipStream_t st) {
    using T = GemmTile<WM, WN, AM, AN>;
    g.tiles_m = (g.M + T::BM - 1) / T::BM;
    g.tiles_n = (g.N + T::BN - 1) / T::BN;
    g.rows_fast = std::min(8, g.tiles_m);
    g.cps = p.cps;
    auto kern = gemm_kernel<DT, WM, WN, AM, AN, Epi>;
    const hipError_t e = ensure_dynamic_lds((const void*)kern, T::kLds);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)((int64_t)g.tiles_m * g.tiles_n * p.splits), T::kThreads, T::kLds, st>>>(g, epi);
    return hipGetLastError();
}

template <int DT, int MODE>
hipError_t launch_store_gemm(const GemmOperands& g, const GemmPlan& p, const StoreArgs<DT>& s, hipStream_t st) {
    return p.big ? launch_gemm<DT, 2, 4, 4, 2>(g, p, StoreEpilogue<DT, MODE, 2, 4, 4, 2>{s}, st)
                 : launch_gemm<DT, 2, 2, 2, 2>(g, p, StoreEpilogue<DT, MODE, 2, 2, 2, 2>{s}, st);
}

template <int DT>
hipError_t launch_store_gemm(const GemmOperands& g, const GemmPlan& p, const StoreArgs<DT>& s, int mode, hipStream_t st) {
    return mode == STORE_OUT   ? launch_store_gemm<DT, STORE_OUT>(g, p, s, st)
           : mode == STORE_SUM ? launch_store_gemm<DT, STORE_SUM>(g, p, s, st)
           : mode == STORE_ADD ? launch_store_gemm<DT, STORE_ADD>(g, p, s, st)
                               : launch_store_gemm<DT, STORE_LAST>(g, p, s, st);
}

// out[m][n] = scale * (sum over the splits, in split order), four values a thread (N a multiple of 8).
template <int DT>
__global__ void __launch_bounds__(256) split_sum_kernel(const float* sum, int splits, int64_t M, int N, uint16_t* out,
                                                        int64_t ldo, const float* scale) {
    const float f = scale ? *scale : 1.0f;
    const int64_t count = M * N;
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < count; i += (int64_t)gridDim.x * 1024) {
        floatx4 v = *reinterpret_cast<const floatx4*>(sum + i);
        for (int z = 1; z < splits; ++z) v += *reinterpret_cast<const floatx4*>(sum + z * count + i);
        const int64_t m = i / N;
        *reinterpret_cast<uint2*>(out + m * ldo + (i - m * N)) =
            make_uint2(f32_to_tile<DT>(v[0] * f) | (uint32_t)f32_to_tile<DT>(v[1] * f) << 16,
                       f32_to_tile<DT>(v[2] * f) | (uint32_t)f32_to_tile<DT>(v[3] * f) << 16);
    }
}

template <int DT>
hipError_t launch_split_sum(const float* sum, int splits, int64_t M, int N, uint16_t* out, int64_t ldo,
                            const float* scale, hipStream_t st) {
    const int64_t blocks = (M * N + 1023) / 1024;
    split_sum_kernel<DT><<<(unsigned)std::min<int64_t>(blocks, 8192), 256, 0, st>>>(sum, splits, M, N, out, ldo, scale);
    return hipGetLastError();
}

}  // namespace aq
