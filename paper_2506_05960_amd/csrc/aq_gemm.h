// Dense 16-bit product on the matrix cores, D = A B^T with fp32 accumulators:
// A [M][K] and B [N][K] row-major (both with K contiguous), and an epilogue
// that consumes a workgroup's D tile in registers.
//
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
__device__ __forceinline__ void gemm_tile(const GemmOperands& g, int& tm, int& tn) {
    const int nwg = (int)gridDim.x, h = (int)blockIdx.x;
    const int xcd = h & 7, j = h >> 3;
    const int per = nwg >> 3, rem = nwg & 7;
    const int w = xcd * per + min(xcd, rem) + j;
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

// D scaled to 16 bits, with an fp32 running sum over several products:
// D + sum -> sum, or, the last time, -> out.
template <int DT, int WM, int WN, int AM, int AN>
struct StoreEpilogue {
    uint16_t* out;         // [M][ldo] the result; null: the sum goes on
    float* sum;            // [M][lds]
    int64_t ldo;
    int first;             // no sum yet
    const float* scale;    // the result times *scale (null: 1)
    __device__ void operator()(const floatx16 (&acc)[AM][AN], int, int m0, int n0, int M, int N, uint8_t*) const {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int wm = wave / WN, wn = wave - wm * WN, l32 = lane & 31, hi = lane >> 5;
        const float f = scale ? *scale : 1.0f;
#pragma unroll
        for (int a = 0; a < AM; ++a)
#pragma unroll
            for (int b = 0; b < AN; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int m = m0 + (wm * AM + a) * 32 + gemm_row(r, hi);
                    const int n = n0 + (wn * AN + b) * 32 + l32;
                    if (m >= M || n >= N) continue;
                    const int64_t i = (int64_t)m * ldo + n;
                    float v = acc[a][b][r];
                    if (!first) v += sum[i];
                    if (out) out[i] = f32_to_tile<DT>(v * f);
                    else sum[i] = v;
                }
    }
};

template <int DT, int WM, int WN, int AM, int AN, class Epi>
__global__ void __launch_bounds__(WM* WN * 64) gemm_kernel(GemmOperands g, Epi epi) {
    using T = GemmTile<WM, WN, AM, AN>;
    extern __shared__ __attribute__((aligned(16))) uint8_t gemm_lds[];
    int tm, tn;
    gemm_tile(g, tm, tn);
    floatx16 acc[AM][AN];
    gemm_mainloop<DT, WM, WN, AM, AN>(g, tm * T::BM, tn * T::BN, 0, (g.K + kGemmChunk - 1) / kGemmChunk, gemm_lds, acc);
    epi(acc, tm, tm * T::BM, tn * T::BN, g.M, g.N, gemm_lds);
}

template <int DT, int WM, int WN, int AM, int AN, class Epi>
hipError_t launch_gemm(GemmOperands g, const Epi& epi, hipStream_t st) {
    using T = GemmTile<WM, WN, AM, AN>;
    g.tiles_m = (g.M + T::BM - 1) / T::BM;
    g.tiles_n = (g.N + T::BN - 1) / T::BN;
    g.rows_fast = std::min(8, g.tiles_m);
    auto kern = gemm_kernel<DT, WM, WN, AM, AN, Epi>;
    const hipError_t e = ensure_dynamic_lds((const void*)kern, T::kLds);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)((int64_t)g.tiles_m * g.tiles_n), T::kThreads, T::kLds, st>>>(g, epi);
    return hipGetLastError();
}

}  // namespace aq
