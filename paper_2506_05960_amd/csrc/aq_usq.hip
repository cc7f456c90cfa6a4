// Linear layers of 4-bit codes with group scales (uniform scalar quantization,
// Sec. 2.3 eq. (3)): entry points and kernels of the forward and the input
// gradient.
//
//     W[i][k] = s[i][j] * (q[i][k] - z[i][j]),   j = k / group
//
// Device layout: codes in tiles of 16 output rows x 128 inputs (1 KiB), the
// 16 bytes of lane l = 16 * o + r holding row r's inputs 32 * s + 8 * o + e of
// step s (word s, value e): word s of all lanes is the B operand of one
// v_mfma_f32_16x16x32 once its eight codes are widened, and a wave reads a tile
// as 64 consecutive 16-byte loads.  Byte b of a word holds value b in its lower
// half and value 4 + b in its upper half.  Scales and zero points:
// [row tile][group][16].
//
// The products run on the codes themselves: integers below 16, exact in fp16
// and bf16, times the unrounded inputs, in fp32.  With S_j the sum of group j's
// inputs,
//     Y[t][i] = sum_j s[i][j] * (sum_{k in j} q[i][k] x[t][k] - z[i][j] * S_j[t]),
// so each group's fp32 sum is scaled once and no weight is ever rounded.
#include <algorithm>
#include <new>
#include <type_traits>

#include "aq_gemm.h"

using aq::api_fail;
using aq::api_hip_fail;

struct aq_usq {
    aq_usq_desc desc;
    int device;
    int nchunk;            // chunks of 128 inputs
    int groups;            // groups a row of the scale array holds (padded to whole chunks)
    uint32_t* d_codes;
    uint16_t* d_scales;
    uint8_t* d_zeros;      // null: every zero point is 8
    uint8_t* d_zero;       // 256 zero bytes
    // more than 64 tokens: group sums of the inputs, and a K split's partial sums
    uint16_t* d_sums;
    float* d_part;
    int sum_groups;
    // input gradient, allocated by its first call
    uint16_t* d_wt;        // [slab][Cp] decoded weights of a slab of inputs, transposed
    float* d_dsum;         // a K split's partial sums
    size_t dsum_bytes, part_bytes;
    uint16_t* d_dy;        // [max_tokens][Cp] output gradient with rows of whole 16-byte groups (C_out % 8 != 0)
    int slab, cp;
};

namespace aq {

namespace {

struct UsqArgs {
    const uint32_t* codes;
    const uint16_t* scales;
    const uint8_t* zeros;
    const uint16_t* X;
    void* Y;
    int y_dtype;
    int n, K, C_out;
    int nchunk, groups;
    int per;               // group >= 128: chunks a group
    // many tokens
    const uint8_t* zero;   // 16 zero bytes
    uint16_t* sums;        // group sums of the inputs
    int sum_groups;        // groups a row of it holds
    float* part;           // K split: [split][n][C_out] partial sums, else null
    int cps;               // chunks a split
};

// (a launch holds fewer than 2^32 threads, and no more than this many blocks of them are of use)
constexpr int64_t kLayoutBlocks = 1 << 20;
unsigned layout_blocks(int64_t count) { return (unsigned)std::min((count + 255) / 256, kLayoutBlocks); }

// Packed codes as the caller has them ([C_out][K / 2], the lower half first) into the device layout.
__global__ void __launch_bounds__(256) usq_pack_kernel(const uint8_t* src, uint32_t* dst, int C_out, int K, int nchunk,
                                                       int64_t words) {
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < words; w += (int64_t)gridDim.x * 256) {
        const int s = (int)(w & 3), lane = (int)(w >> 2) & 63;
        const int64_t tile = w >> 8;
        const int c = (int)(tile % nchunk);
        const int64_t i = tile / nchunk * 16 + (lane & 15);
        const int k = c * 128 + s * 32 + (lane >> 4) * 8;
        uint32_t v = 0, o = 0;
        if (i < C_out && k < K) v = *reinterpret_cast<const uint32_t*>(src + i * (K / 2) + k / 2);
#pragma unroll
        for (int e = 0; e < 8; ++e) o |= ((v >> (4 * e)) & 15u) << (8 * (e & 3) + 4 * (e >> 2));
        dst[w] = o;
    }
}

// [C_out][G] -> [row tile][groups][16], zero past the ends.
template <typename T>
__global__ void __launch_bounds__(256) usq_groups_kernel(const T* src, T* dst, int C_out, int G, int groups, int64_t count) {
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < count; w += (int64_t)gridDim.x * 256) {
        const int64_t i = w / (16 * (int64_t)groups) * 16 + (w & 15);
        const int j = (int)(w / 16 % groups);
        dst[w] = i < C_out && j < G ? src[i * G + j] : T(0);
    }
}

// The eight codes of a word as 16-bit floats in value order.  A byte b below 16
// is the fp8 (e4m3) number b * 2^-9, subnormal or not, so the conversion from
// fp8 with the scale 2^9 widens two codes an instruction, exactly (all sixteen
// codes checked): 7 instructions a word.  Through fp32, byte by byte, it
// takes 15.
template <int DT>
__device__ __forceinline__ u32x4 widen_codes(uint32_t w) {
    const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
    u32x4 o;
    if constexpr (DT == AQ_F16) {
        o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false));
        o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true));
        o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false));
        o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true));
    } else {
        o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false));
        o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true));
        o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false));
        o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true));
    }
    return o;
}

template <int DT>
__device__ __forceinline__ floatx4 mfma16(const u32x4& a, const u32x4& b, const floatx4& c) {
    if constexpr (DT == AQ_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0,
                                                      0, 0);
}

template <int DT>
__device__ __forceinline__ float widen16(uint16_t b) {
    if constexpr (DT == AQ_BF16) return bf16_to_f32(b);
    else return f16_to_f32(b);
}

__device__ __forceinline__ void store_y3(void* Y, int y_dtype, int64_t i, float v) {
    if (y_dtype == AQ_F32) static_cast<float*>(Y)[i] = v;
    else if (y_dtype == AQ_F16) static_cast<uint16_t*>(Y)[i] = f32_to_f16(v);
    else static_cast<uint16_t*>(Y)[i] = f32_to_bf16(v);
}

// ---- few tokens ----

constexpr int kFewTokens = 64;

// 16 RT output rows x 16 NT tokens a workgroup; its waves share K chunk by
// chunk and add their sums in LDS in wave order.  SG: steps of 32 inputs a
// scale group (group 32, 64, and 128 or more).  S_j comes from a product with
// ones, which delivers it in the accumulators' own layout.
//  * STAGE false (up to four tokens): the tokens are read in the operands' own
//    layout, and a wave has U chunks' loads on their way at a time.
//  * STAGE true: that layout puts neighbouring lanes on different tokens, and a
//    load of sixteen tokens then takes a cycle a lane.  The tokens reach a
//    buffer of the wave's own in LDS in runs of 64 bytes instead (four lanes a
//    token, pieces permuted so that sixteen tokens' reads lie in different
//    banks), a chunk ahead: four times as fast.
template <int DT, int SG, int NT, int RT, int U, int WAVES, bool STAGE>
__global__ void __launch_bounds__(WAVES * 64) usq_few_kernel(UsqArgs a) {
    static_assert(!STAGE || U == 1, "one chunk ahead");
    constexpr int GPC = 4 / SG;
    extern __shared__ __attribute__((aligned(16))) uint8_t few_lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const int l16 = lane & 15, o = lane >> 4;
    const int tiles = (a.C_out + 15) >> 4;
    const u32x4* codes[RT];
    int64_t srow[RT];
#pragma unroll
    for (int y = 0; y < RT; ++y) {
        const int64_t rt = min((int)blockIdx.x * RT + y, tiles - 1);      // (a repeated tile's rows are not stored)
        codes[y] = reinterpret_cast<const u32x4*>(a.codes) + rt * a.nchunk * 64 + lane;
        srow[y] = rt * a.groups * 16 + l16;
    }
    const uint32_t one = DT == AQ_BF16 ? 0x3f803f80u : 0x3c003c00u;
    const u32x4 ones{one, one, one, one};
    floatx4 acc[RT][NT];
#pragma unroll
    for (int y = 0; y < RT; ++y)
#pragma unroll
        for (int m = 0; m < NT; ++m) acc[y][m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

    u32x4 w[U][RT];
    uint16_t sc[U][RT][GPC], zp[U][RT][GPC];
    auto load_weights = [&](int u, int c) {
#pragma unroll
        for (int y = 0; y < RT; ++y) {
            w[u][y] = codes[y][(int64_t)c * 64];
#pragma unroll
            for (int g = 0; g < GPC; ++g) {
                const int64_t at = srow[y] + (int64_t)(GPC == 1 ? c / a.per : c * GPC + g) * 16;
                sc[u][y][g] = a.scales[at];
                zp[u][y][g] = a.zeros ? a.zeros[at] : 8;
            }
        }
    };
    // one chunk's products: its codes, scales and zero points, and its tokens
    auto chunk = [&](const u32x4 (&cw)[RT], const uint16_t (&cs)[RT][GPC], const uint16_t (&cz)[RT][GPC],
                     const u32x4 (&xv)[4][NT]) {
#pragma unroll
        for (int g = 0; g < GPC; ++g) {
            floatx4 xs[NT];
#pragma unroll
            for (int m = 0; m < NT; ++m) {
                xs[m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = g * SG; s < (g + 1) * SG; ++s) xs[m] = mfma16<DT>(xv[s][m], ones, xs[m]);
            }
#pragma unroll
            for (int y = 0; y < RT; ++y) {
                floatx4 d[NT];
#pragma unroll
                for (int m = 0; m < NT; ++m) d[m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = g * SG; s < (g + 1) * SG; ++s) {
                    const u32x4 q = widen_codes<DT>(cw[y][s]);
#pragma unroll
                    for (int m = 0; m < NT; ++m) d[m] = mfma16<DT>(xv[s][m], q, d[m]);
                }
                const float sf = widen16<DT>(cs[y][g]), z = (float)cz[y][g];
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[y][m][r] = __builtin_fmaf(sf, __builtin_fmaf(-z, xs[m][r], d[m][r]), acc[y][m][r]);
            }
        }
    };

    if constexpr (STAGE) {
        uint8_t* buf = few_lds + wave * NT * 4096;      // [token block][step][token][four pieces of 16 bytes]
        const int tok = lane >> 2, piece = (lane & 3) ^ ((tok >> 2) & 3);
        const __amdgpu_buffer_rsrc_t rx = buffer_rsrc(a.X, 0xFFFFFFFFu);
        uint32_t ox[NT];
#pragma unroll
        for (int m = 0; m < NT; ++m) ox[m] = ((uint32_t)min(16 * m + tok, a.n - 1) * (uint32_t)a.K + 8u * piece) * 2u;
        auto issue = [&](int c) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int m = 0; m < NT; ++m) {
                    uint8_t* dst = buf + (m * 4 + s) * 1024;
                    const int k = c * 128 + 32 * s;
                    if (c * 128 + 128 <= a.K) {
                        lds_dma16(rx, ox[m], (uint32_t)k * 2u, dst);
                    } else {
                        const uint8_t* p = reinterpret_cast<const uint8_t*>(a.X + k) + ox[m];
                        lds_dma16(k + 8 * piece < a.K ? p : a.zero, dst);
                    }
                }
        };
        const uint32_t at = (uint32_t)(l16 * 64 + ((o ^ ((l16 >> 2) & 3)) * 16));
        if (wave < a.nchunk) {
            issue(wave);
            load_weights(0, wave);
        }
        for (int c = wave; c < a.nchunk; c += waves) {
            wait_vmcnt<0>();
            u32x4 xv[4][NT], cw[RT];
            uint16_t cs[RT][GPC], cz[RT][GPC];
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int m = 0; m < NT; ++m) xv[s][m] = *reinterpret_cast<const u32x4*>(buf + (m * 4 + s) * 1024 + at);
#pragma unroll
            for (int y = 0; y < RT; ++y) {
                cw[y] = w[0][y];
#pragma unroll
                for (int g = 0; g < GPC; ++g) {
                    cs[y][g] = sc[0][y][g];
                    cz[y][g] = zp[0][y][g];
                }
            }
            if (c + waves < a.nchunk) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // the buffer is read: the next chunk may land
                issue(c + waves);
                load_weights(0, c + waves);
            }
            chunk(cw, cs, cz, xv);
        }
        __syncthreads();                                // the buffers become the sums' below
    } else {
        const uint16_t* x[NT];
#pragma unroll
        for (int m = 0; m < NT; ++m) x[m] = a.X + (int64_t)min(16 * m + l16, a.n - 1) * a.K + 8 * o;
        for (int c0 = wave; c0 < a.nchunk; c0 += U * waves) {
            u32x4 xv[U][4][NT];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = c0 + u * waves;
                load_weights(u, min(c, a.nchunk - 1));
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const int k = c * 128 + 32 * s;
#pragma unroll
                    for (int m = 0; m < NT; ++m) {
                        xv[u][s][m] = u32x4{0, 0, 0, 0};                   // past K (and past the last chunk): nothing
                        if (k + 8 * o < a.K) xv[u][s][m] = *reinterpret_cast<const u32x4*>(x[m] + k);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) chunk(w[u], sc[u], zp[u], xv[u]);
        }
    }
    floatx4* red = reinterpret_cast<floatx4*>(few_lds);      // [wave][row tile][token block][lane]
#pragma unroll
    for (int y = 0; y < RT; ++y)
#pragma unroll
        for (int m = 0; m < NT; ++m) red[((wave * RT + y) * NT + m) * 64 + lane] = acc[y][m];
    __syncthreads();
    for (int ym = wave; ym < RT * NT; ym += waves) {
        floatx4 v = red[ym * 64 + lane];
        for (int w = 1; w < waves; ++w) v += red[(w * RT * NT + ym) * 64 + lane];
        const int rt = blockIdx.x * RT + ym / NT, i = rt * 16 + l16;
        if (i >= a.C_out) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int tok = 16 * (ym % NT) + 4 * o + r;
            if (tok < a.n) store_y3(a.Y, a.y_dtype, (int64_t)tok * a.C_out + i, v[r]);
        }
    }
}

template <int DT, int SG, int NT, int RT, int U, int WAVES, bool STAGE>
hipError_t launch_few(const UsqArgs& a, hipStream_t st) {
    const unsigned grid = (unsigned)((a.C_out + 16 * RT - 1) / (16 * RT));
    const int waves = std::min(WAVES, a.nchunk);
    const size_t lds = (size_t)waves * NT * std::max(STAGE ? 4096 : 0, RT * 1024);
    auto kern = usq_few_kernel<DT, SG, NT, RT, U, WAVES, STAGE>;
    const hipError_t e = ensure_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<grid, waves * 64, lds, st>>>(a);
    return hipGetLastError();
}

// Output rows a workgroup (16 RT).  Compute units that take a second workgroup take twice the time, so two row tiles
// share a workgroup, and the tokens' reads, where there are more than 256 of them, and four where there are more than
// 512 (groups of 128 and more: finer ones have too many values to hold for 64 tokens).  us, RT = 1 / 2 / 4, row tiles
// in front:
//   K 4096, group 128, 24 tokens:  256  6.2 / 6.9 / 9.2    288  8.5 / 7.0 / 9.1     512  9.3 / 8.2 / 10.6    576 11.1 / 11.3 / 10.6
//                      64 tokens:  256 11.2 / 10.6 / 14.3  288 17.8 / 10.9 / 14.4   512 20.8 / 14.0 / 16.3   576 27.1 / 22.1 / 16.4
//   K 2304, group 32,  24 tokens:  256  5.8 / 6.7 / 9.9    288  7.3 / 6.7 / 9.9     512  8.2 / 7.2 / 10.1    576 10.9 / 11.7 / 10.1
//                      48 tokens:  256  8.8 / 9.7          288 14.9 / 9.9           512 16.5 / 10.9          576 22.0 / 18.9
// Up to 16 tokens two tiles at most, and short reductions not before there are more than 768 of them:
//   K 8192, 1 token:   256 6.4 / 7.6    288 8.6 / 7.7    576 11.5 / 11.1    1024 15.2 / 12.8
//   K 4096, 1 token:   256 4.9 / 4.9    288 5.3 / 4.9    448  5.6 / 5.1     1024  9.0 / 7.2
//   K 2304, 1 token:   288 5.1 / 5.4    576 5.2 / 5.5    768  5.3 / 5.4      896  6.5 / 5.6
// Long reductions in up to 256 row tiles take sixteen waves: K 8192, 1 token, 128 tiles 5.7 -> 5.3, 256 6.4 -> 5.7.
template <int DT, int SG>
hipError_t launch_few(const UsqArgs& a, hipStream_t st) {
    constexpr int kUnits = 256;
    const int tiles = (a.C_out + 15) / 16;
    const bool one = tiles <= kUnits, two = tiles <= 2 * kUnits;
    if (a.n <= 16) {
        const bool wide = (!one && a.nchunk >= 32) || tiles > 3 * kUnits, deep = one && a.nchunk >= 64;
        if (a.n <= 4)
            return wide   ? launch_few<DT, SG, 1, 2, 2, 8, false>(a, st)
                   : deep ? launch_few<DT, SG, 1, 1, 2, 16, false>(a, st)
                          : launch_few<DT, SG, 1, 1, 2, 8, false>(a, st);
        return wide   ? launch_few<DT, SG, 1, 2, 1, 8, true>(a, st)
               : deep ? launch_few<DT, SG, 1, 1, 1, 16, true>(a, st)
                      : launch_few<DT, SG, 1, 1, 1, 8, true>(a, st);
    }
    if (a.n <= 32)
        return one   ? launch_few<DT, SG, 2, 1, 1, 8, true>(a, st)
               : two ? launch_few<DT, SG, 2, 2, 1, 8, true>(a, st)
                     : launch_few<DT, SG, 2, 4, 1, 8, true>(a, st);
    if constexpr (SG == 4)
        if (!two) return launch_few<DT, SG, 4, 4, 1, 8, true>(a, st);
    return one ? launch_few<DT, SG, 4, 1, 1, 8, true>(a, st) : launch_few<DT, SG, 4, 2, 1, 8, true>(a, st);
}

// ---- many tokens ----

// Group sums of the inputs, S[t][j], as three bf16 pieces that add up to the
// fp32 sum: [group][n][8] = {h, m, l, h, m, l, 0, 0}.
template <int DT>
__global__ void __launch_bounds__(256) usq_sums_kernel(UsqArgs a, int group) {
    // eight lanes a group, 16-byte loads
    const int gp = a.sum_groups;
    const int part = threadIdx.x & 7;
    for (int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3; id < (int64_t)a.n * gp; id += (int64_t)gridDim.x * 32) {
        const int64_t t = id / gp;
        const int j = (int)(id - t * gp);
        float s = 0.0f;
        for (int k = j * group + 8 * part; k < min((j + 1) * group, a.K); k += 64) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(a.X + t * a.K + k);
#pragma unroll
            for (int e = 0; e < 4; ++e) s += widen16<DT>((uint16_t)v[e]) + widen16<DT>((uint16_t)(v[e] >> 16));
        }
        s += __shfl_xor(s, 1);
        s += __shfl_xor(s, 2);
        s += __shfl_xor(s, 4);
        if (part != 0) continue;
        const uint32_t h = f32_to_bf16(s);
        const float r1 = s - bf16_to_f32((uint16_t)h);
        const uint32_t m = f32_to_bf16(r1);
        const uint32_t l = f32_to_bf16(r1 - bf16_to_f32((uint16_t)m));
        reinterpret_cast<u32x4*>(a.sums)[(int64_t)j * a.n + t] = u32x4{h | m << 16, l | h << 16, m | l << 16, 0u};
    }
}

// WM x WN waves (four) on a tile of 32 WM AM tokens x 32 WN AN output rows, each
// on 32 AM x 32 AN of it in blocks of v_mfma_f32_32x32x16 (D rows: tokens,
// columns: output rows, so that a lane has one scale a block and group).
// Launched as 1 x 4 waves on 128 x 128: every wave all of the tile's tokens, so
// that no two waves widen the same codes.
//  * The tile's tokens reach LDS 128 inputs at a time through direct-to-LDS
//    loads, in two stages (slots permuted as in gemm_mainloop, sixteen a row).
//  * Weights go from the code tiles to registers, are widened there once a
//    chunk, and serve all of the wave's tokens; no LDS traffic.
//  * A group's sum accumulates on its own (AM x AN independent chains) and is
//    scaled into the running sum.
//  * The zero points come first: -s z times the group sums is a product over
//    groups, of s z in two bf16 pieces (15 bits at most, exact) and the sums in
//    three, six of the eight values a lane holds for one group.
// A chunk takes a wave 32 matrix instructions (1024 cycles of its SIMD's matrix
// core) and some 200 vector ones (800 cycles; 56 widen, 64 scale, the rest are
// moves, addresses and the tile's ends).  4096 x 4096 -> 4096 bf16, group 128:
// 154 us, 0.89 PFLOP/s; counters at 2.0 GHz: the matrix cores are busy for 48 %
// of the time, the vector ALUs for 36 %, and the two waves of a SIMD hardly
// overlap one with the other.
// SG: steps of 16 inputs a group within a chunk.
template <int DT, int SG, int WM, int WN, int AM, int AN>
__global__ void __launch_bounds__(256, 2) usq_gemm_kernel(UsqArgs a) {
    constexpr int BM = 32 * WM * AM, BN = 32 * WN * AN;
    static_assert(WM * WN == 4, "four waves");
    constexpr int STAGE = BM * 256, LOADS = BM * 16 / 256;
    extern __shared__ __attribute__((aligned(16))) uint8_t usq_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave - wm * WN, l32 = lane & 31, hi = lane >> 5;
    // XCD-aware order: each XCD takes a contiguous run, token tiles fastest in bands of eight
    const int tiles_m = (a.n + BM - 1) / BM, tiles_n = (a.C_out + BN - 1) / BN;
    int tm, tn, z;
    {
        const int nwg = (int)gridDim.x, h = (int)blockIdx.x;
        const int xcd = h & 7, per = nwg >> 3, rem = nwg & 7;
        int w = xcd * per + min(xcd, rem) + (h >> 3);
        z = w / (tiles_m * tiles_n);
        w -= z * tiles_m * tiles_n;
        const int band = w / (8 * tiles_n), rows = min(8, tiles_m - 8 * band);
        const int in = w - band * 8 * tiles_n;
        tn = in / rows;
        tm = 8 * band + in - tn * rows;
    }
    const int m0 = tm * BM, n0 = tn * BN;
    const int c_beg = z * a.cps, c_end = min(a.nchunk, c_beg + a.cps);

    // ---- staging of the tokens ----
    const int r0 = tid >> 4, slot = (tid & 15) ^ (r0 & 15);
    // a whole chunk through buffer loads (the row's offset in a register, the chunk's in a scalar), the last
    // part of a chunk through addresses that point past K's end at the zero block
    const uint16_t* tx = a.X + (int64_t)m0 * a.K;
    const __amdgpu_buffer_rsrc_t rx = buffer_rsrc(tx, 0xFFFFFFFFu);
    const int mx = min(BM, a.n - m0) - 1;
    uint32_t ox[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) ox[j] = (uint32_t)(min(r0 + 16 * j, mx) * a.K + 8 * slot) * 2u;
    auto issue = [&](int chunk, uint8_t* st) {
        const int k0 = chunk * 128;
        if (k0 + 128 <= a.K) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) lds_dma16(rx, ox[j], (uint32_t)k0 * 2u, st + (j * 256 + wave * 64) * 16);
        } else {
            const bool in = k0 + 8 * slot < a.K;
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
                lds_dma16(in ? reinterpret_cast<const uint8_t*>(tx + k0) + ox[j] : a.zero,
                          st + (j * 256 + wave * 64) * 16);
        }
    };

    // ---- weights: this lane's column of each block, two 16-byte loads a chunk ----
    const u32x4* pc[AN];
    int64_t srow[AN];
#pragma unroll
    for (int b = 0; b < AN; ++b) {
        const int i = n0 + (wn * AN + b) * 32 + l32;
        const int rt = min(i, a.C_out - 1) >> 4;       // rows past the end: any tile, never stored
        pc[b] = reinterpret_cast<const u32x4*>(a.codes) + (int64_t)rt * a.nchunk * 64 + 16 * hi + (i & 15);
        srow[b] = (int64_t)rt * a.groups * 16 + (i & 15);
    }
    constexpr int GPC = 8 / SG;                        // groups a chunk (1 for groups of 128 and more)
    u32x4 wc[AN][2];
    uint16_t sc[AN][GPC];
    auto load_weights = [&](int chunk) {
#pragma unroll
        for (int b = 0; b < AN; ++b) {
            wc[b][0] = pc[b][(int64_t)chunk * 64];
            wc[b][1] = pc[b][(int64_t)chunk * 64 + 32];
#pragma unroll
            for (int g = 0; g < GPC; ++g) {
                const int j = GPC == 1 ? chunk / a.per : chunk * GPC + g;
                sc[b][g] = a.scales[srow[b] + (int64_t)j * 16];
            }
        }
    };

    floatx16 acc[AM][AN];
#pragma unroll
    for (int x = 0; x < AM; ++x)
#pragma unroll
        for (int b = 0; b < AN; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[x][b][r] = 0.0f;

    issue(c_beg, usq_lds);
    load_weights(c_beg);
    u32x4 w[AN][2];              // the chunk's codes and scales, while the next one's are loaded
    float s32[AN][GPC];
    auto take_weights = [&]() {
#pragma unroll
        for (int b = 0; b < AN; ++b) {
            w[b][0] = wc[b][0];
            w[b][1] = wc[b][1];
#pragma unroll
            for (int g = 0; g < GPC; ++g) s32[b][g] = widen16<DT>(sc[b][g]);
        }
    };
    // ---- zero points of the groups that begin in this split's chunks ----
    {
        const int j_beg = GPC == 1 ? (c_beg + a.per - 1) / a.per : c_beg * GPC;
        const int j_end = GPC == 1 ? (c_end + a.per - 1) / a.per : c_end * GPC;
        const u32x4* ps[AM];
#pragma unroll
        for (int x = 0; x < AM; ++x)
            ps[x] = reinterpret_cast<const u32x4*>(a.sums) + min(m0 + (wm * AM + x) * 32 + l32, a.n - 1);
#pragma unroll 4
        for (int j0 = j_beg; j0 < j_end; j0 += 2) {
            const int j = min(j0 + hi, j_end - 1);
            const bool live = j0 + hi < j_end;
            u32x4 fs[AM];
#pragma unroll
            for (int x = 0; x < AM; ++x) {
                fs[x] = ps[x][(int64_t)min(j, a.sum_groups - 1) * a.n];
                if (!live) fs[x] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int b = 0; b < AN; ++b) {
                const int64_t at = srow[b] + (int64_t)j * 16;
                const float v = -widen16<DT>(a.scales[at]) * (a.zeros ? (float)a.zeros[at] : 8.0f);
                const uint32_t h = f32_to_bf16(v), l = f32_to_bf16(v - bf16_to_f32((uint16_t)h));
                const u32x4 fz{h | h << 16, h | l << 16, l | l << 16, 0u};
#pragma unroll
                for (int x = 0; x < AM; ++x) acc[x][b] = mfma_gemm<AQ_BF16>(fs[x], fz, acc[x][b]);
            }
        }
    }

    // ---- products ----
    // Step u + 1's operands are read and widened between step u's products; a chunk's last step multiplies
    // behind the barrier that hands its stage over; and a group's sum is scaled into the running sum
    // between the first products of the next group, block by block.
    const uint32_t arow = (uint32_t)(wm * AM * 32 + l32) * 256u;
    u32x4 xf[2][AM], q[2][AN];
    auto operand = [&](const uint8_t* st, int u, int i) {
        if (i < AM)
            xf[u & 1][i] = *reinterpret_cast<const u32x4*>(st + arow + i * 8192 + (((2 * u + hi) ^ (l32 & 15)) * 16));
        else q[u & 1][i - AM] = widen_codes<DT>(w[i - AM][u & 1][u >> 1]);
    };
    floatx16 d[AM][AN];
    float sprev[AN];
#pragma unroll
    for (int b = 0; b < AN; ++b) sprev[b] = 0.0f;
#pragma unroll
    for (int x = 0; x < AM; ++x)
#pragma unroll
        for (int b = 0; b < AN; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) d[x][b][r] = 0.0f;
    auto scale = [&](int x, int b) {
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[x][b][r] = __builtin_fmaf(sprev[b], d[x][b][r], acc[x][b][r]);
    };
    wait_vmcnt<0>();
    lds_barrier();
    take_weights();
    if (c_beg + 1 < c_end) {
        issue(c_beg + 1, usq_lds + STAGE);
        load_weights(c_beg + 1);
    }
#pragma unroll
    for (int i = 0; i < AM + AN; ++i) operand(usq_lds, 0, i);
    constexpr int kOps = AM + AN, kProducts = AM * AN;
    for (int c = c_beg; c < c_end; ++c) {
        uint8_t* st = usq_lds + ((c - c_beg) & 1) * STAGE;
        const uint8_t* next = usq_lds + ((c + 1 - c_beg) & 1) * STAGE;
        float snext[AN][GPC];
#pragma unroll
        for (int b = 0; b < AN; ++b)
#pragma unroll
            for (int g = 0; g < GPC; ++g) snext[b][g] = s32[b][g];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (u == 7 && c + 1 < c_end) {
                wait_vmcnt<0>();     // this wave's part of chunk c + 1 landed, its codes too
                lds_barrier();       // everyone's; and every wave has read all of chunk c
                take_weights();
                if (c + 2 < c_end) {
                    issue(c + 2, st);
                    load_weights(c + 2);
                }
            }
#pragma unroll
            for (int i = 0; i < kProducts; ++i) {
                // (the last chunk's reads of the other stage are not used)
#pragma unroll
                for (int o = 2 * i; o < (i + 1 == kProducts ? kOps : min(2 * i + 2, kOps)); ++o)
                    operand(u < 7 ? st : next, (u + 1) & 7, o);
                const int x = i / AN, b = i % AN;
                if (u % SG == 0) {
                    scale(x, b);
                    asm volatile("" : "+v"(acc[x][b]));      // before the group's sum is overwritten
                    floatx16 zero;
#pragma unroll
                    for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
                    d[x][b] = mfma_gemm<DT>(xf[u & 1][x], q[u & 1][b], zero);
                } else {
                    d[x][b] = mfma_gemm<DT>(xf[u & 1][x], q[u & 1][b], d[x][b]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (u % SG == 0) {
#pragma unroll
                for (int b = 0; b < AN; ++b) sprev[b] = snext[b][u / SG];
            }
        }
    }
#pragma unroll
    for (int x = 0; x < AM; ++x)
#pragma unroll
        for (int b = 0; b < AN; ++b) scale(x, b);

    // branch-free buffer stores at offsets from the tile's corner (past the edge: past the buffer)
    auto store = [&](void* base, auto bytes, auto&& put) {
        constexpr int kBytes = decltype(bytes)::value;
        const __amdgpu_buffer_rsrc_t ry =
            buffer_rsrc(static_cast<uint8_t*>(base) + ((int64_t)m0 * a.C_out + n0) * kBytes, kOutOfRange);
#pragma unroll
        for (int x = 0; x < AM; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int t = (wm * AM + x) * 32 + gemm_row(r, hi);
#pragma unroll
                for (int b = 0; b < AN; ++b) {
                    const int i = (wn * AN + b) * 32 + l32;
                    const bool in = m0 + t < a.n && n0 + i < a.C_out;
                    put(ry, in ? (uint32_t)(t * a.C_out + i) * (uint32_t)kBytes : kOutOfRange, acc[x][b][r]);
                }
            }
    };
    auto put32 = [](__amdgpu_buffer_rsrc_t ry, uint32_t off, float v) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), ry, off, 0, 0);
    };
    using four = std::integral_constant<int, 4>;
    using two = std::integral_constant<int, 2>;
    if (a.part) store(a.part + (int64_t)z * a.n * a.C_out, four{}, put32);
    else if (a.y_dtype == AQ_F32) store(a.Y, four{}, put32);
    else if (a.y_dtype == AQ_F16) store(a.Y, two{}, [](__amdgpu_buffer_rsrc_t ry, uint32_t off, float v) {
        __builtin_amdgcn_raw_buffer_store_b16(f32_to_f16(v), ry, off, 0, 0);
    });
    else store(a.Y, two{}, [](__amdgpu_buffer_rsrc_t ry, uint32_t off, float v) {
        __builtin_amdgcn_raw_buffer_store_b16(f32_to_bf16(v), ry, off, 0, 0);
    });
}

// Y = sum over the K splits, in split order.
__global__ void __launch_bounds__(256) usq_join_kernel(const float* part, int splits, int64_t count, void* Y, int y_dtype) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        float v = part[i];
        for (int z = 1; z < splits; ++z) v += part[z * count + i];
        store_y3(Y, y_dtype, i, v);
    }
}

struct UsqPlan {
    int tiles, splits, cps;
};

// K splits of a call, shortest by a model fitted to measured ones (4096 -> 4096, us with 1 / 2 / 3 / 4 / 8 splits:
// 128 tokens 48 / 31 / 26 / 26 / 28, 256 tokens 49 / 35 / 31 / 34 / 37, 1024 tokens 59 / 54 / - / - / -; 16384 ->
// 4096, 128 tokens 194 / 103 / 73 / 58 / 39): a workgroup's fixed time, its time a chunk alone on its compute unit or
// with a second one (more of it the smaller the groups), and the partial sums written and read back.  `cap`: bytes
// there are for them.
UsqPlan usq_plan(int64_t n, int C_out, int nchunk, int group, size_t cap) {
    const int64_t tiles = (n + 127) / 128 * ((C_out + 127) / 128);
    const double small = group == 32 ? 1.6 : group == 64 ? 1.2 : 1.0;
    UsqPlan best{(int)tiles, 1, nchunk};
    double best_us = 1e30;
    for (int s = 1; s <= std::max(1, nchunk / 2) && tiles * s <= std::max<int64_t>(tiles, 512); ++s) {
        if (s > 1 && (size_t)s * n * C_out * 4 > cap) break;
        const int cps = (nchunk + s - 1) / s;
        if ((nchunk + cps - 1) / cps != s) continue;
        const int64_t wgs = tiles * s;
        const double work = wgs <= 256 ? 5.0 + (1.4 + wgs * 0.001) * small * cps
                                       : (double)((wgs + 511) / 512) * (5.0 + 2.3 * small * cps);
        const double us = work + (s > 1 ? s * (1.0 + 1.3e-6 * n * C_out) : 0.0);
        if (us < best_us) {
            best_us = us;
            best.splits = s;
            best.cps = cps;
        }
    }
    return best;
}

template <int DT, int SG, int WM, int WN, int AM, int AN>
hipError_t launch_usq_gemm(const UsqArgs& a, int grid, hipStream_t st) {
    constexpr size_t lds = 2 * 32 * WM * AM * 256;
    auto kern = usq_gemm_kernel<DT, SG, WM, WN, AM, AN>;
    const hipError_t e = ensure_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<(unsigned)grid, 256, lds, st>>>(a);
    return hipGetLastError();
}

template <int DT, int SG>
hipError_t launch_many(UsqArgs a, int group, float* part, size_t part_bytes, hipStream_t st) {
    const UsqPlan p = usq_plan(a.n, a.C_out, a.nchunk, group, part_bytes);
    const int64_t blocks = ((int64_t)a.n * a.sum_groups * 8 + 255) / 256;
    usq_sums_kernel<DT><<<(unsigned)std::min<int64_t>(blocks, 1 << 20), 256, 0, st>>>(a, group);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.cps = p.cps;
    a.part = p.splits > 1 ? part : nullptr;
    e = launch_usq_gemm<DT, SG, 1, 4, 4, 1>(a, p.tiles * p.splits, st);
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t count = (int64_t)a.n * a.C_out;
    usq_join_kernel<<<(unsigned)std::min<int64_t>((count + 255) / 256, 4096), 256, 0, st>>>(part, p.splits, count, a.Y,
                                                                                           a.y_dtype);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_usq_forward(const UsqArgs& a, int group, float* part, size_t pb, hipStream_t st) {
    if (a.n <= kFewTokens)
        return group == 32 ? launch_few<DT, 1>(a, st) : group == 64 ? launch_few<DT, 2>(a, st) : launch_few<DT, 4>(a, st);
    return group == 32   ? launch_many<DT, 2>(a, group, part, pb, st)
           : group == 64 ? launch_many<DT, 4>(a, group, part, pb, st)
                         : launch_many<DT, 8>(a, group, part, pb, st);
}

// ---- input gradient ----

// Wt[k - k0][i] of the chunk of 128 inputs blockIdx.x and 64 output rows
// blockIdx.y, rounded once to 16 bits; rows of output channels past C_out are
// zeros (their scales are).  Bound by memory and by the 2-byte writes that
// transpose in LDS: 4096 x 8192 bf16 18 us, 84 MB at 4.7 TB/s.
template <int DT>
__global__ void __launch_bounds__(256) usq_decode_t_kernel(UsqArgs a, int group, int c0, uint16_t* wt, int cp) {
    __shared__ __attribute__((aligned(16))) uint16_t tile[128][72];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = c0 + blockIdx.x, rt = blockIdx.y * 4 + wave;
    const int l16 = lane & 15, o = lane >> 4;
    const bool live = rt * 16 < a.C_out;
    u32x4 w{0, 0, 0, 0};
    if (live) w = reinterpret_cast<const u32x4*>(a.codes)[((int64_t)rt * a.nchunk + c) * 64 + lane];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int k = 32 * s + 8 * o;
        float sc = 0.0f, z = 8.0f;
        if (live) {
            const int64_t at = ((int64_t)rt * a.groups + (c * 128 + k) / group) * 16 + l16;
            sc = widen16<DT>(a.scales[at]);
            if (a.zeros) z = (float)a.zeros[at];
        }
        const u32x4 v = widen_codes<DT>(w[s]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float q = widen16<DT>((uint16_t)(v[e >> 1] >> (16 * (e & 1))));
            tile[k + e][16 * wave + l16] = f32_to_tile<DT>(sc * (q - z));
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int k = (threadIdx.x >> 3) + 32 * j, i = 8 * (threadIdx.x & 7);
        const int col = blockIdx.y * 64 + i;
        if (col < cp)
            *reinterpret_cast<u32x4*>(wt + (int64_t)(blockIdx.x * 128 + k) * cp + col) =
                *reinterpret_cast<const u32x4*>(&tile[k][i]);
    }
}

// Few tokens: the chunk of 128 inputs blockIdx.x of dX, summed over the rows of
// split blockIdx.y, without W in memory.  A wave decodes 32 output rows x 128
// inputs (rounded once to 16 bits, as above) into an LDS buffer of its own, and
// transposing reads deliver them with the rows as the summed index.  The waves
// add their sums in LDS in wave order, the splits through split_sum_kernel.
// Bound by the decode (fp32 per weight) and, with the tokens, by the loads of dY,
// whose lanes lie on different tokens, and the splits' sums.
// SG: steps of 32 inputs a scale group, as in usq_few_kernel.
constexpr int kGradRows = 32, kGradPitch = 272;     // a row's 256 bytes and 16: rows start in different banks
template <int DT, int SG, int NT>
__global__ void __launch_bounds__(256) usq_few_grad_kernel(UsqArgs a, const uint16_t* dy, int cp, int rows_split, float* sum) {
    constexpr int GPC = 4 / SG, WAVES = 4, kBuf = kGradRows * kGradPitch;
    static_assert(kBuf >= 8 * 64 * 16, "a wave's buffer holds its sums of 16 tokens");
    __shared__ __attribute__((aligned(16))) uint8_t lds[WAVES * kBuf];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, o = lane >> 4, c = (int)blockIdx.x;
    const int tiles = (a.C_out + 15) >> 4;
    const int r_beg = (int)blockIdx.y * rows_split, r_end = min(cp, r_beg + rows_split);
    uint8_t* buf = lds + wave * kBuf;
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)buf;
    uint32_t at[2][4];         // this lane's place in row 8 o + l16 / 4 of the blocks of 16 inputs
#pragma unroll
    for (int i = 0; i < 8; ++i)
        at[i >> 2][i & 3] = base + (uint32_t)((8 * o + (l16 >> 2)) * kGradPitch + i * 32 + (l16 & 3) * 8);
    const uint16_t* y[NT];
#pragma unroll
    for (int m = 0; m < NT; ++m) y[m] = dy + (int64_t)min(16 * m + l16, a.n - 1) * cp;
    floatx4 acc[NT][8];
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[m][i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

    u32x4 w[2], yv[NT];
    uint16_t sc[2][GPC], zp[2][GPC];
    auto load = [&](int r) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t rt = min((r >> 4) + t, tiles - 1);     // (a repeated tile's rows meet zeros of dY)
            w[t] = reinterpret_cast<const u32x4*>(a.codes)[(rt * a.nchunk + c) * 64 + lane];
#pragma unroll
            for (int g = 0; g < GPC; ++g) {
                const int64_t p = (rt * a.groups + (GPC == 1 ? c / a.per : c * GPC + g)) * 16 + l16;
                sc[t][g] = a.scales[p];
                zp[t][g] = a.zeros ? a.zeros[p] : 8;
            }
        }
#pragma unroll
        for (int m = 0; m < NT; ++m) {
            yv[m] = u32x4{0, 0, 0, 0};
            if (r + 8 * o < r_end) yv[m] = *reinterpret_cast<const u32x4*>(y[m] + r + 8 * o);
        }
    };
    int r = r_beg + wave * kGradRows;
    if (r < r_end) load(r);
    for (; r < r_end; r += WAVES * kGradRows) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const float f = widen16<DT>(sc[t][s / SG]), z = (float)zp[t][s / SG];
                const u32x4 q = widen_codes<DT>(w[t][s]);
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = f32_to_tile<DT>(f * (widen16<DT>((uint16_t)q[e]) - z)) |
                           (uint32_t)f32_to_tile<DT>(f * (widen16<DT>((uint16_t)(q[e] >> 16)) - z)) << 16;
                *reinterpret_cast<u32x4*>(buf + (16 * t + l16) * kGradPitch + 64 * s + 16 * o) = v;
            }
        u32x4 x[NT];
#pragma unroll
        for (int m = 0; m < NT; ++m) x[m] = yv[m];
        if (r + WAVES * kGradRows < r_end) load(r + WAVES * kGradRows);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 b[4];       // (the wave's own writes come before its reads: LDS serves a wave in order)
            lds_read_tr<0, kGradPitch, kGradPitch>(at[h], b);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int m = 0; m < NT; ++m) acc[m][4 * h + i] = mfma16<DT>(x[m], b[i], acc[m][4 * h + i]);
        }
    }
    floatx4* red = reinterpret_cast<floatx4*>(lds);       // [wave][block of 16 inputs][lane]
#pragma unroll
    for (int m = 0; m < NT; ++m) {
        __syncthreads();      // the buffers, or the last tokens' sums, are read
#pragma unroll
        for (int i = 0; i < 8; ++i) red[(wave * 8 + i) * 64 + lane] = acc[m][i];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = wave + 4 * j, k = c * 128 + 16 * i + l16;
            floatx4 v = red[i * 64 + lane];
#pragma unroll
            for (int q = 1; q < WAVES; ++q) v += red[(q * 8 + i) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = 16 * m + 4 * o + e;
                if (k < a.K && t < a.n) sum[((int64_t)blockIdx.y * a.n + t) * a.K + k] = v[e];
            }
        }
    }
}

// Rows a split: whole steps of the four waves; splits for one workgroup a compute unit, or two of layers that leave
// them four steps each, within `cap` bytes of sums.  us with 256 / 512 / 1024 workgroups: 4096 -> 4096, 1 token 10.6 /
// 10.5 / 11.5, 16 tokens 11.6 / 12.3 / 15.0, 64 tokens 17.5 / 21.9 / 27.6; 4096 -> 16384, 1 token 24.9 / 21.5 / 20.8,
// 64 tokens 32.3 / 31.6 / 38.7 (through W in memory 27 to 32 and 58 to 60).
int few_grad_rows(int n, int K, int cp, size_t cap) {
    const int chunks = (K + 127) / 128, steps = (cp + 4 * kGradRows - 1) / (4 * kGradRows);
    const int64_t fit = (int64_t)(cap / ((size_t)n * K * 4));
    const int wgs = (int64_t)steps * chunks >= 2048 ? 512 : 256;
    const int splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(steps, fit), wgs / chunks));
    return (steps + splits - 1) / splits * 4 * kGradRows;
}

template <int DT, int SG>
hipError_t launch_few_grad(const UsqArgs& a, const uint16_t* dy, int cp, float* sum, size_t cap, uint16_t* dX, hipStream_t st) {
    const int rows = few_grad_rows(a.n, a.K, cp, cap), splits = (cp + rows - 1) / rows;
    const dim3 grid((unsigned)((a.K + 127) / 128), (unsigned)splits);
    if (a.n <= 16) usq_few_grad_kernel<DT, SG, 1><<<grid, 256, 0, st>>>(a, dy, cp, rows, sum);
    else if (a.n <= 32) usq_few_grad_kernel<DT, SG, 2><<<grid, 256, 0, st>>>(a, dy, cp, rows, sum);
    else usq_few_grad_kernel<DT, SG, 4><<<grid, 256, 0, st>>>(a, dy, cp, rows, sum);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_split_sum<DT, false>(sum, splits, a.n, a.K, dX, a.K, nullptr, nullptr, st);
}

// dst[r][c] of pitch cp = src[r][c], zero for C <= c < cp.
__global__ void __launch_bounds__(256) pad_rows_kernel(const uint16_t* src, int C, uint16_t* dst, int cp) {
    const int64_t r = blockIdx.y;
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < cp) dst[r * cp + c] = c < C ? src[r * C + c] : 0;
}

template <int DT>
hipError_t input_grad(const aq_usq* L, const UsqArgs& a, const uint16_t* dY, uint16_t* dX, int n, hipStream_t st) {
    const int K = a.K, C = a.C_out, cp = L->cp;
    hipError_t e;
    GemmOperands g{};
    g.zero = L->d_zero;
    g.A = dY;
    if (C % 8 != 0) {
        for (int r = 0; r < n; r += 65535) {
            const int rows = std::min(65535, n - r);
            pad_rows_kernel<<<dim3((unsigned)((cp + 255) / 256), (unsigned)rows), 256, 0, st>>>(
                dY + (int64_t)r * C, C, L->d_dy + (int64_t)r * cp, cp);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        g.A = L->d_dy;
    }
    if (n <= kFewTokens && (size_t)n * K * 4 <= L->dsum_bytes) {
        const auto dy = static_cast<const uint16_t*>(g.A);
        return L->desc.group == 32   ? launch_few_grad<DT, 1>(a, dy, cp, L->d_dsum, L->dsum_bytes, dX, st)
               : L->desc.group == 64 ? launch_few_grad<DT, 2>(a, dy, cp, L->d_dsum, L->dsum_bytes, dX, st)
                                     : launch_few_grad<DT, 4>(a, dy, cp, L->d_dsum, L->dsum_bytes, dX, st);
    }
    g.lda = g.ldb = g.K = cp;
    g.M = n;
    g.B = L->d_wt;
    for (int k0 = 0; k0 < K; k0 += L->slab) {
        const int cols = std::min(L->slab, K - k0);
        usq_decode_t_kernel<DT><<<dim3((unsigned)((cols + 127) / 128), (unsigned)((cp + 63) / 64)), 256, 0, st>>>(
            a, L->desc.group, k0 / 128, L->d_wt, cp);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        g.N = cols;
        const GemmPlan p = gemm_plan(n, cols, cp, L->dsum_bytes);
        const StoreArgs<DT> s{dX + k0, L->d_dsum, K, nullptr, nullptr};
        e = p.splits > 1 ? launch_store_gemm<DT, false, STORE_SUM>(g, p, s, st)
                         : launch_store_gemm<DT, false, STORE_OUT>(g, p, s, st);
        if (e != hipSuccess) return e;
        if (p.splits > 1 &&
            (e = launch_split_sum<DT, false>(L->d_dsum, p.splits, n, cols, dX + k0, K, nullptr, nullptr, st)) != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace

}  // namespace aq

namespace {

void free_usq(aq_usq* L) {
    void* ptrs[] = {L->d_codes, L->d_scales, L->d_zeros, L->d_zero, L->d_sums, L->d_part, L->d_wt, L->d_dsum, L->d_dy};
    for (void* p : ptrs)
        if (p) (void)hipFree(p);
    delete L;
}

template <typename T>
aq_status alloc(T** p, size_t bytes, const char* what) {
    if (*p) return AQ_OK;
    const hipError_t e = hipMalloc(reinterpret_cast<void**>(p), bytes);
    if (e == hipSuccess) return AQ_OK;
    *p = nullptr;
    return api_hip_fail(e, what);
}

bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

constexpr size_t kPartBytes = size_t(32) << 20;    // most that the forward's K splits take
constexpr size_t kSplitBytes = size_t(64) << 20;   // and the input gradient's

// Weights into the device layout, through a staging buffer that is freed again.
aq_status upload(aq_usq* L, const void* codes, const void* scales, const uint8_t* zeros) {
    const aq_usq_desc& d = L->desc;
    const int64_t tiles = (d.out_features + 15) / 16;
    const int G = (int)((d.in_features + (int64_t)d.group - 1) / d.group);
    const size_t code_bytes = (size_t)d.out_features * (d.in_features / 2), group_count = (size_t)d.out_features * G;
    const int64_t words = tiles * L->nchunk * 256, count = tiles * L->groups * 16;
    aq_status s = alloc(&L->d_codes, (size_t)words * 4, "codes");
    if (s == AQ_OK) s = alloc(&L->d_scales, (size_t)count * 2, "scales");
    if (s == AQ_OK && zeros) s = alloc(&L->d_zeros, (size_t)count, "zero points");
    if (s == AQ_OK) s = alloc(&L->d_zero, 256, "zero block");
    if (s == AQ_OK && d.max_tokens > aq::kFewTokens) {
        L->sum_groups = G;
        s = alloc(&L->d_sums, (size_t)d.max_tokens * L->sum_groups * 16, "group sums");
        // (fewer tokens of the same tiles never split less: each step of 128 is bounded by its first token's splits)
        size_t need = 0;
        for (int64_t lo = 1; lo <= d.max_tokens && lo <= 128 * 512; lo += 128) {
            const aq::UsqPlan p = aq::usq_plan(lo, d.out_features, L->nchunk, d.group, kPartBytes);
            if (p.splits > 1) need = std::max(need, (size_t)p.splits * std::min(lo + 127, d.max_tokens) * d.out_features * 4);
        }
        need = std::min(need, kPartBytes);
        if (s == AQ_OK && need) s = alloc(&L->d_part, need, "partial sums");
        if (s == AQ_OK) L->part_bytes = need;
    }
    uint8_t* tmp = nullptr;
    if (s == AQ_OK) s = alloc(&tmp, std::max(code_bytes, group_count * 2), "staging buffer");
    if (s != AQ_OK) return s;
    hipError_t e = hipMemset(L->d_zero, 0, 256);
    if (e == hipSuccess) e = hipMemcpy(tmp, codes, code_bytes, hipMemcpyHostToDevice);
    if (e == hipSuccess) {
        aq::usq_pack_kernel<<<aq::layout_blocks(words), 256, 0, nullptr>>>(tmp, L->d_codes, d.out_features,
                                                                          d.in_features, L->nchunk, words);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e == hipSuccess) e = hipMemcpy(tmp, scales, group_count * 2, hipMemcpyHostToDevice);
    const unsigned blocks = aq::layout_blocks(count);
    if (e == hipSuccess) {
        aq::usq_groups_kernel<uint16_t><<<blocks, 256, 0, nullptr>>>(reinterpret_cast<const uint16_t*>(tmp), L->d_scales,
                                                                   d.out_features, G, L->groups, count);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e == hipSuccess && zeros) {
        e = hipMemcpy(tmp, zeros, group_count, hipMemcpyHostToDevice);
        if (e == hipSuccess) {
            aq::usq_groups_kernel<uint8_t><<<blocks, 256, 0, nullptr>>>(tmp, L->d_zeros, d.out_features, G, L->groups,
                                                                      count);
            e = hipGetLastError();
        }
        if (e == hipSuccess) e = hipDeviceSynchronize();
    }
    (void)hipFree(tmp);
    return e == hipSuccess ? AQ_OK : api_hip_fail(e, "weight layout");
}

aq_status check_call(const aq_usq* L, const void* in, const void* out, int64_t n) {
    if (!L || !in || !out) return api_fail(AQ_ERR_INVALID_ARGUMENT, "null pointer argument");
    if (n < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "n must be >= 1");
    if (n > L->desc.max_tokens) return api_fail(AQ_ERR_INVALID_ARGUMENT, "tokens exceed max_tokens");
    if (misaligned(in) || misaligned(out))
        return api_fail(AQ_ERR_INVALID_ARGUMENT, "inputs and outputs must be 16-byte aligned");
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return api_hip_fail(e, "hipGetDevice");
    if (dev != L->device) return api_fail(AQ_ERR_INVALID_ARGUMENT, "layer created on another device");
    const int64_t wide = std::max(L->desc.in_features, L->desc.out_features);
    if ((n + 127) / 128 * ((wide + 127) / 128) > aq::kMaxTiles)
        return api_fail(AQ_ERR_UNSUPPORTED, "too many tokens times features for one call");
    return AQ_OK;
}

aq::UsqArgs make_args(const aq_usq* L, const void* X, void* Y, int64_t n) {
    return aq::UsqArgs{L->d_codes, L->d_scales, L->d_zeros, static_cast<const uint16_t*>(X), Y, L->desc.y_dtype,
                       (int)n, L->desc.in_features, L->desc.out_features, L->nchunk, L->groups,
                       std::max(1, L->desc.group / 128), L->d_zero, L->d_sums, L->sum_groups, nullptr, 0};
}

}  // namespace

extern "C" {

aq_status aq_usq_create(const aq_usq_desc* desc, const void* codes, const void* scales, const uint8_t* zeros,
                        aq_usq** out) {
    if (out) *out = nullptr;
    if (!desc || !codes || !scales || !out) return api_fail(AQ_ERR_INVALID_ARGUMENT, "null pointer argument");
    const aq_usq_desc& d = *desc;
    if (d.out_features < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "out_features must be >= 1");
    if (d.in_features < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "in_features must be >= 1");
    if (d.group < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "group must be >= 1");
    if (d.dtype < AQ_F32 || d.dtype > AQ_I8) return api_fail(AQ_ERR_INVALID_ARGUMENT, "bad dtype");
    if (d.y_dtype < AQ_F32 || d.y_dtype > AQ_BF16) return api_fail(AQ_ERR_INVALID_ARGUMENT, "y_dtype must be F32, F16 or BF16");
    if (d.max_tokens < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "max_tokens must be >= 1");
    if (d.dtype != AQ_F16 && d.dtype != AQ_BF16)
        return api_fail(AQ_ERR_UNSUPPORTED, "4-bit layers take fp16 or bf16 inputs and scales");
    if (d.in_features % 8 != 0) return api_fail(AQ_ERR_UNSUPPORTED, "in_features must be a multiple of 8");
    if (d.group != 32 && d.group != 64 && d.group % 128 != 0)
        return api_fail(AQ_ERR_UNSUPPORTED, "group must be 32, 64 or a multiple of 128");
    if (d.in_features > aq::kMaxPitch || d.out_features > aq::kMaxPitch || d.max_tokens > (1 << 24))
        return api_fail(AQ_ERR_UNSUPPORTED, "features above 2^21 or max_tokens above 2^24");
    if (zeros) {
        const int64_t count = (int64_t)d.out_features * ((d.in_features + (int64_t)d.group - 1) / d.group);
        for (int64_t i = 0; i < count; ++i)
            if (zeros[i] > 15) return api_fail(AQ_ERR_INVALID_ARGUMENT, "zero point above 15");
    }
    int ndev = 0;
    hipError_t e = hipGetDeviceCount(&ndev);
    if (e != hipSuccess || ndev < 1) return api_fail(AQ_ERR_DEVICE, "no HIP device available");
    aq_usq* L = new (std::nothrow) aq_usq();
    if (!L) return api_fail(AQ_ERR_OUT_OF_MEMORY, "host allocation");
    L->desc = d;
    e = hipGetDevice(&L->device);
    if (e != hipSuccess) {
        delete L;
        return api_hip_fail(e, "hipGetDevice");
    }
    L->nchunk = (d.in_features + 127) / 128;
    L->groups = d.group < 128 ? L->nchunk * (128 / d.group) : (L->nchunk + d.group / 128 - 1) / (d.group / 128);
    const aq_status s = upload(L, codes, scales, zeros);
    if (s != AQ_OK) {
        free_usq(L);
        return s;
    }
    *out = L;
    return AQ_OK;
}

aq_status aq_usq_forward(aq_usq* L, const void* X, void* Y, int64_t n, void* stream) {
    const aq_status s = check_call(L, X, Y, n);
    if (s != AQ_OK) return s;
    const aq::UsqArgs a = make_args(L, X, Y, n);
    const auto st = static_cast<hipStream_t>(stream);
    const hipError_t e = L->desc.dtype == AQ_F16 ? aq::launch_usq_forward<AQ_F16>(a, L->desc.group, L->d_part, L->part_bytes, st)
                                                 : aq::launch_usq_forward<AQ_BF16>(a, L->desc.group, L->d_part, L->part_bytes, st);
    return e == hipSuccess ? AQ_OK : api_hip_fail(e, "forward launch");
}

aq_status aq_usq_input_grad(aq_usq* L, const void* dY, void* dX, int64_t n, void* stream) {
    aq_status s = check_call(L, dY, dX, n);
    if (s != AQ_OK) return s;
    const int C = L->desc.out_features;
    if (!L->cp) {
        L->cp = (C + 7) / 8 * 8;
        // Slabs of equal width and of at most 128 MiB, whole tiles of the product: the fewer there are the fewer of
        // their products need K splits to fill the chip (4096 x 8192 -> 4096, two of 32 MiB 284 us, one 243; 64 tokens,
        // 4096 -> 16384, four 124 us, one 60).
        const int64_t padded = (int64_t)L->nchunk * 128, most = std::max<int64_t>(256, (int64_t(64) << 20) / L->cp);
        const int64_t slabs = (padded + most - 1) / most;
        L->slab = (int)std::min(padded, ((padded + slabs - 1) / slabs + 255) / 256 * 256);
    }
    // W goes through memory for more than 64 tokens, and where the sums of the most few tokens do not fit
    const int K = L->desc.in_features, few = (int)std::min<int64_t>(L->desc.max_tokens, aq::kFewTokens);
    const size_t one = (size_t)few * K * 4;
    const bool slabs = L->desc.max_tokens > aq::kFewTokens || one > kSplitBytes;
    if (((slabs && !L->d_wt) || !L->d_dsum || (C % 8 != 0 && !L->d_dy)) && aq::capturing(static_cast<hipStream_t>(stream)))
        return api_fail(AQ_ERR_UNSUPPORTED, "the first input gradient allocates: not under graph capture");
    if (slabs) s = alloc(&L->d_wt, (size_t)L->slab * L->cp * 2, "gradient workspace");
    if (s == AQ_OK && !L->d_dsum) {
        size_t bytes = 16;
        if (slabs) {
            const int cols = std::min(L->slab, K), tail = K % L->slab;
            bytes = std::max(bytes, aq::gemm_split_bytes(L->desc.max_tokens, cols, L->cp, kSplitBytes));
            if (tail) bytes = std::max(bytes, aq::gemm_split_bytes(L->desc.max_tokens, tail, L->cp, kSplitBytes));
        }
        if (one <= kSplitBytes) {
            const int rows = aq::few_grad_rows(few, K, L->cp, kSplitBytes);
            bytes = std::max(bytes, one * ((L->cp + rows - 1) / rows));
        }
        s = alloc(&L->d_dsum, bytes, "gradient workspace");
        if (s == AQ_OK) L->dsum_bytes = bytes;
    }
    if (s == AQ_OK && C % 8 != 0) s = alloc(&L->d_dy, (size_t)L->desc.max_tokens * L->cp * 2, "gradient workspace");
    if (s != AQ_OK) return s;
    const aq::UsqArgs a = make_args(L, nullptr, nullptr, n);
    const auto dy = static_cast<const uint16_t*>(dY);
    const auto dx = static_cast<uint16_t*>(dX);
    const auto st = static_cast<hipStream_t>(stream);
    const hipError_t e = L->desc.dtype == AQ_F16 ? aq::input_grad<AQ_F16>(L, a, dy, dx, (int)n, st)
                                                 : aq::input_grad<AQ_BF16>(L, a, dy, dx, (int)n, st);
    return e == hipSuccess ? AQ_OK : api_hip_fail(e, "input gradient launch");
}

aq_status aq_usq_destroy(aq_usq* L) {
    if (!L) return AQ_OK;
    const hipError_t e = hipDeviceSynchronize();
    free_usq(L);
    return e == hipSuccess ? AQ_OK : api_hip_fail(e, "destroy");
}

}  // extern "C"
