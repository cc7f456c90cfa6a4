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
// as 64 consecutive 16-byte loads.  Value 2 p of a word is its nibble p and
// value 2 p + 1 its nibble p + 4, so that one shift and mask leaves a pair in
// the two halves of a register.  Scales and zero points: [row tile][group][16].
//
// q - z is an integer of five bits, exact in fp16 and bf16: the matrix cores
// multiply it with the unrounded inputs, and the scale is applied to each
// group's fp32 sum.  No weight is rounded.
#include <algorithm>
#include <new>

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
    // input gradient, allocated by its first call
    uint16_t* d_wt;        // [slab][Cp] decoded weights of a slab of inputs, transposed
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
};

// Packed codes as the caller has them ([C_out][K / 2], the lower half first) into the device layout.
__global__ void __launch_bounds__(256) usq_pack_kernel(const uint8_t* src, uint32_t* dst, int C_out, int K, int nchunk,
                                                       int64_t words) {
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w >= words) return;
    const int s = (int)(w & 3), lane = (int)(w >> 2) & 63;
    const int64_t tile = w >> 8;
    const int c = (int)(tile % nchunk);
    const int64_t i = tile / nchunk * 16 + (lane & 15);
    const int k = c * 128 + s * 32 + (lane >> 4) * 8;
    uint32_t v = 0, o = 0;
    if (i < C_out && k < K) v = *reinterpret_cast<const uint32_t*>(src + i * (K / 2) + k / 2);
#pragma unroll
    for (int p = 0; p < 4; ++p) o |= ((v >> (8 * p)) & 15u) << (4 * p) | ((v >> (8 * p + 4)) & 15u) << (4 * p + 16);
    dst[w] = o;
}

// [C_out][G] -> [row tile][groups][16], zero past the ends.
template <typename T>
__global__ void __launch_bounds__(256) usq_groups_kernel(const T* src, T* dst, int C_out, int G, int groups, int64_t count) {
    const int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (w >= count) return;
    const int64_t i = w / (16 * (int64_t)groups) * 16 + (w & 15);
    const int j = (int)(w / 16 % groups);
    dst[w] = i < C_out && j < G ? src[i * G + j] : T(0);
}

// The eight codes of a word as 16-bit integers in value order.
template <int DT>
__device__ __forceinline__ u32x4 widen_codes(uint32_t w) {
    u32x4 o;
    if constexpr (DT == AQ_F16) {
        // 0x6400 | q is 1024 + q
        const half2v off{(_Float16)-1024.0f, (_Float16)-1024.0f};
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const uint32_t v = ((w >> (4 * p)) & 0x000f000fu) | 0x64006400u;
            o[p] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, v) + off);
        }
    } else {
        const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
        // an integer below 16 fills the upper half of its fp32 alone
        auto pair = [](uint32_t b, int x, int y) {
            const uint32_t fx = __float_as_uint((float)((b >> (8 * x)) & 255u));
            const uint32_t fy = __float_as_uint((float)((b >> (8 * y)) & 255u));
            return __builtin_amdgcn_perm(fy, fx, 0x07060302u);
        };
        o[0] = pair(lo, 0, 2);
        o[1] = pair(hi, 0, 2);
        o[2] = pair(lo, 1, 3);
        o[3] = pair(hi, 1, 3);
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

// 16 output rows x 16 tokens a workgroup; its waves share K chunk by chunk and
// add their sums in LDS in wave order.  SG: steps of 32 inputs a scale group
// (group 32, 64, and 128 or more).  The zero point leaves through the group
// sum of the inputs, z * sum_k x, which a product with ones delivers in the
// accumulators' own layout.
template <int DT, int SG>
__global__ void __launch_bounds__(512) usq_few_kernel(UsqArgs a) {
    __shared__ floatx4 red[8][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6;
    const int l16 = lane & 15, o = lane >> 4;
    const int rt = blockIdx.x, t0 = blockIdx.y * 16;
    const int t = min(t0 + l16, a.n - 1);
    const uint16_t* x = a.X + (int64_t)t * a.K + 8 * o;
    const u32x4* codes = reinterpret_cast<const u32x4*>(a.codes) + (int64_t)rt * a.nchunk * 64 + lane;
    const int64_t srow = (int64_t)rt * a.groups * 16 + l16;
    const uint32_t one = DT == AQ_BF16 ? 0x3f803f80u : 0x3c003c00u;
    const u32x4 ones{one, one, one, one};
    floatx4 acc{0.0f, 0.0f, 0.0f, 0.0f};
    for (int c = wave; c < a.nchunk; c += waves) {
        const u32x4 w = codes[(int64_t)c * 64];
        u32x4 xv[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int k = c * 128 + 32 * s;
            xv[s] = u32x4{0, 0, 0, 0};
            if (k + 8 * o < a.K) xv[s] = *reinterpret_cast<const u32x4*>(x + k);
        }
#pragma unroll
        for (int g = 0; g < 4 / SG; ++g) {
            const int j = SG == 4 ? c / a.per : c * (4 / SG) + g;
            const float sc = widen16<DT>(a.scales[srow + (int64_t)j * 16]);
            const float z = a.zeros ? (float)a.zeros[srow + (int64_t)j * 16] : 8.0f;
            floatx4 d{0.0f, 0.0f, 0.0f, 0.0f}, xs{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = g * SG; s < (g + 1) * SG; ++s) {
                d = mfma16<DT>(xv[s], widen_codes<DT>(w[s]), d);
                xs = mfma16<DT>(xv[s], ones, xs);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(sc, __builtin_fmaf(-z, xs[r], d[r]), acc[r]);
        }
    }
    red[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < waves; ++w) acc += red[w][lane];
    const int i = rt * 16 + l16;
    if (i >= a.C_out) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int tok = t0 + 4 * o + r;
        if (tok < a.n) store_y3(a.Y, a.y_dtype, (int64_t)tok * a.C_out + i, acc[r]);
    }
}

template <int DT, int SG>
hipError_t launch_few(const UsqArgs& a, hipStream_t st) {
    const int waves = std::min(8, a.nchunk);
    constexpr int kMost = 65535 * 16;          // tokens of a launch
    for (int t0 = 0; t0 < a.n; t0 += kMost) {
        UsqArgs p = a;
        p.n = std::min(kMost, a.n - t0);
        p.X += (int64_t)t0 * a.K;
        p.Y = static_cast<uint8_t*>(a.Y) + (int64_t)t0 * a.C_out * (a.y_dtype == AQ_F32 ? 4 : 2);
        usq_few_kernel<DT, SG><<<dim3((unsigned)((a.C_out + 15) / 16), (unsigned)((p.n + 15) / 16)), waves * 64, 0, st>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int DT>
hipError_t launch_usq_forward(const UsqArgs& a, int group, hipStream_t st) {
    return group == 32 ? launch_few<DT, 1>(a, st) : group == 64 ? launch_few<DT, 2>(a, st) : launch_few<DT, 4>(a, st);
}

// ---- input gradient ----

// Wt[k - k0][i] of the chunk of 128 inputs blockIdx.x and 64 output rows
// blockIdx.y, rounded once to 16 bits; rows of output channels past C_out are
// zeros (their scales are).
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

// dst[r][c] of pitch cp = src[r][c], zero for C <= c < cp.
__global__ void __launch_bounds__(256) pad_rows_kernel(const uint16_t* src, int C, uint16_t* dst, int cp) {
    const int64_t r = blockIdx.y;
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c < cp) dst[r * cp + c] = c < C ? src[r * C + c] : 0;
}

template <int DT>
hipError_t input_grad(const aq_usq* L, const UsqArgs& a, const uint16_t* dY, uint16_t* dX, int n, hipStream_t st) {
    constexpr int WM = 2, WN = 4, AM = 4, AN = 2;
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
    g.lda = C % 8 ? cp : C;
    g.M = n;
    g.B = L->d_wt;
    g.ldb = cp;
    g.K = C % 8 ? cp : C;
    for (int k0 = 0; k0 < K; k0 += L->slab) {
        const int cols = std::min(L->slab, K - k0);
        usq_decode_t_kernel<DT><<<dim3((unsigned)((cols + 127) / 128), (unsigned)((cp + 63) / 64)), 256, 0, st>>>(
            a, L->desc.group, k0 / 128, L->d_wt, cp);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        g.N = cols;
        StoreEpilogue<DT, WM, WN, AM, AN> se{dX + k0, nullptr, K, 1, nullptr};
        if ((e = launch_gemm<DT, WM, WN, AM, AN>(g, se, st)) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

}  // namespace aq

namespace {

void free_usq(aq_usq* L) {
    void* ptrs[] = {L->d_codes, L->d_scales, L->d_zeros, L->d_zero, L->d_wt, L->d_dy};
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

// Weights into the device layout, through a staging buffer that is freed again.
aq_status upload(aq_usq* L, const void* codes, const void* scales, const uint8_t* zeros) {
    const aq_usq_desc& d = L->desc;
    const int64_t tiles = (d.out_features + 15) / 16;
    const int G = (d.in_features + d.group - 1) / d.group;
    const size_t code_bytes = (size_t)d.out_features * (d.in_features / 2), group_count = (size_t)d.out_features * G;
    const int64_t words = tiles * L->nchunk * 256, count = tiles * L->groups * 16;
    aq_status s = alloc(&L->d_codes, (size_t)words * 4, "codes");
    if (s == AQ_OK) s = alloc(&L->d_scales, (size_t)count * 2, "scales");
    if (s == AQ_OK && zeros) s = alloc(&L->d_zeros, (size_t)count, "zero points");
    if (s == AQ_OK) s = alloc(&L->d_zero, 256, "zero block");
    uint8_t* tmp = nullptr;
    if (s == AQ_OK) s = alloc(&tmp, std::max(code_bytes, group_count * 2), "staging buffer");
    if (s != AQ_OK) return s;
    hipError_t e = hipMemset(L->d_zero, 0, 256);
    if (e == hipSuccess) e = hipMemcpy(tmp, codes, code_bytes, hipMemcpyHostToDevice);
    if (e == hipSuccess) {
        aq::usq_pack_kernel<<<(unsigned)((words + 255) / 256), 256, 0, nullptr>>>(tmp, L->d_codes, d.out_features,
                                                                                 d.in_features, L->nchunk, words);
        e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e == hipSuccess) e = hipMemcpy(tmp, scales, group_count * 2, hipMemcpyHostToDevice);
    const unsigned blocks = (unsigned)((count + 255) / 256);
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
    return AQ_OK;
}

aq::UsqArgs make_args(const aq_usq* L, const void* X, void* Y, int64_t n) {
    return aq::UsqArgs{L->d_codes, L->d_scales, L->d_zeros, static_cast<const uint16_t*>(X), Y, L->desc.y_dtype,
                       (int)n, L->desc.in_features, L->desc.out_features, L->nchunk, L->groups,
                       std::max(1, L->desc.group / 128)};
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
    if (d.in_features > (1 << 24) || d.out_features > (1 << 24) || d.max_tokens > (1 << 24))
        return api_fail(AQ_ERR_UNSUPPORTED, "sizes above 2^24");
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
    const hipError_t e = L->desc.dtype == AQ_F16 ? aq::launch_usq_forward<AQ_F16>(a, L->desc.group, st)
                                                 : aq::launch_usq_forward<AQ_BF16>(a, L->desc.group, st);
    return e == hipSuccess ? AQ_OK : api_hip_fail(e, "forward launch");
}

aq_status aq_usq_input_grad(aq_usq* L, const void* dY, void* dX, int64_t n, void* stream) {
    aq_status s = check_call(L, dY, dX, n);
    if (s != AQ_OK) return s;
    const int C = L->desc.out_features;
    if (!L->cp) {
        L->cp = (C + 7) / 8 * 8;
        const int64_t most = std::max<int64_t>(128, (int64_t(16) << 20) / L->cp / 128 * 128);   // 32 MiB
        L->slab = (int)std::min<int64_t>(most, (int64_t)L->nchunk * 128);
    }
    s = alloc(&L->d_wt, (size_t)L->slab * L->cp * 2, "gradient workspace");
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
