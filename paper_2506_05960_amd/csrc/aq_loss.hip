// Losses over a vocabulary and their gradients: distillation from a teacher's
// top logits, and softmax cross entropy of a head's logits without keeping the
// logits.  Entry points and kernels.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "aq_gemm.h"

using aq::api_fail;
using aq::api_hip_fail;

struct aq_loss {
    aq_loss_desc desc;
    int device;
    int piece;             // cross entropy: vocabulary rows a piece of the gradient covers
    uint8_t* d_zero;       // 256 zero bytes
    float2* d_seg;         // distillation of few rows: [row][segment] maximum and sum of exponentials
    float* d_list;         // and [row][top] the listed tokens' logits
    float2* d_part;        // [vocabulary tile of 128][max_tokens] maximum and sum of exponentials
    float* d_row;          // [max_tokens] x {target logit, maximum, log2 of the sum, row weight, peak}, then the call's peak
    // gradient workspace, allocated by the first call that needs it
    uint16_t* d_dlt;       // [piece][tokens] logits' gradient of a piece
    uint16_t* d_dlx;       // the same scaled token by token (fp16, for dX beside dW)
    uint16_t* d_xt;        // [features][tokens] inputs, transposed
    float* d_dx;           // [split][tokens][features] input gradient of the pieces so far
    size_t dx_bytes;
};

namespace aq {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kMaxTop = 1024;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// (m, s) of two disjoint parts of a row: maximum, and sum of 2^(c (z - m)).
__device__ __forceinline__ void merge(float& m, float& s, float om, float os, float c) {
    const float nm = fmaxf(m, om);
    const float b = nm == -INFINITY ? 0.0f : nm;    // nothing finite yet: both sums are zero
    s = s * exp2_fast((m - b) * c) + os * exp2_fast((om - b) * c);
    m = nm;
}

// ---- distillation ----

template <int DT>
struct Store {
    static constexpr int kVec = DT == AQ_F32 ? 4 : 8;   // values of 16 bytes
};

template <int DT>
__device__ __forceinline__ void unpack(const u32x4& v, float (&o)[Store<DT>::kVec]) {
    if constexpr (DT == AQ_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __uint_as_float(v[e]);
    } else if constexpr (DT == AQ_BF16) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[2 * e] = __uint_as_float(v[e] << 16);
            o[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[2 * e] = f16_to_f32((uint16_t)v[e]);
            o[2 * e + 1] = f16_to_f32((uint16_t)(v[e] >> 16));
        }
    }
}

template <int DT>
__device__ __forceinline__ u32x4 pack(const float (&o)[Store<DT>::kVec]) {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (DT == AQ_F32) v[e] = __float_as_uint(o[e]);
        else v[e] = (uint32_t)f32_to_tile<DT>(o[2 * e]) | (uint32_t)f32_to_tile<DT>(o[2 * e + 1]) << 16;
    }
    return v;
}

template <int DT>
__device__ __forceinline__ void store_as(void* p, int64_t i, float v) {
    if constexpr (DT == AQ_F32) static_cast<float*>(p)[i] = v;
    else static_cast<uint16_t*>(p)[i] = f32_to_tile<DT>(v);
}

struct DistillArgs {
    const void* logits;
    const int32_t* ids;
    const void* teacher;
    const float* dloss;
    float* loss;
    void* grad;
    int64_t n;
    int V, top;
    float c;               // log2(e) / temperature
    float T;
    // rows in segments, a workgroup each
    int segs, seg_vecs;    // segments a row, 16-byte vectors a segment
    float2* part;          // [row][segment]
    float* list;           // [row][top] the listed tokens' logits (the gradient may overwrite the logits)
};

enum DistillPart {
    DISTILL_ROW,           // a whole row: statistics, loss and gradient
    DISTILL_STATS,         // a segment's maximum and sum
    DISTILL_GRAD           // the loss, and a segment's gradient
};

// One workgroup a row, or a segment of one.  The first NV 16-byte vectors of each thread stay in registers between the
// statistics and the gradient; a longer row's others are read twice.  Bound by memory: what is read or
// written for the last time passes the caches by (non-temporal), so that the second reads find theirs there
// (4096 x 131072 bf16: 542 -> 513 us, with rolled loops 502, 4.3 TB/s of the 2.1 GB that cannot be done without).
template <int DT, int THREADS, int NV, DistillPart PART>
__device__ __forceinline__ void distill_row(const DistillArgs& a, const int64_t row, const int seg) {
    constexpr int VEC = Store<DT>::kVec;
    constexpr int WAVES = THREADS / 64;
    __shared__ float s_m[WAVES], s_s[WAVES];
    __shared__ float s_t[kMaxTop], s_z[kMaxTop];       // the list's teacher and student logits
    __shared__ int32_t s_id[kMaxTop];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int V = a.V, top = a.top;
    const int64_t base = row * V;
    const int head = min(V, (int)((VEC - base % VEC) % VEC));
    const int nvec = (V - head) / VEC;
    const int tail0 = head + nvec * VEC;
    // this workgroup's vectors; the first one takes what lies before and behind the row's
    const int v0 = PART == DISTILL_ROW ? 0 : min(nvec, seg * a.seg_vecs);
    const int v1 = PART == DISTILL_ROW ? nvec : min(nvec, v0 + a.seg_vecs);
    const bool first = PART == DISTILL_ROW || seg == 0;
    const bool lists = PART != DISTILL_STATS || first, reads = PART != DISTILL_GRAD || a.grad;
    const u32x4* body = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.logits) +
                                                       (base + head) * (16 / VEC));
    // the list first: its logits wait for its ids
    int32_t id0 = -1;
    float t0 = -INFINITY;
    if (lists && tid < top) {
        id0 = a.ids[row * top + tid];
        t0 = load_as_f32<DT>(a.teacher, row * top + tid);
    }
    const float dloss = a.dloss ? a.dloss[row] : 1.0f;
    u32x4 held[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (reads && v0 + tid + i * THREADS < v1) {
            const u32x4* p = &body[v0 + tid + i * THREADS];
            held[i] = PART == DISTILL_STATS ? *p : __builtin_nontemporal_load(p);
        }
    // values before and behind the whole vectors: one a thread
    const int edge = !first ? -1 : tid < head ? tid : tid < head + V - tail0 ? tail0 + tid - head : -1;
    const float zedge = edge >= 0 ? load_as_f32<DT>(a.logits, base + edge) : -INFINITY;
    bool bad = false;                       // an id past the vocabulary
#pragma unroll 1
    for (int j = lists ? tid : top; j < top; j += THREADS) {
        int32_t id = id0;
        float t = t0;
        if (j != tid) {
            id = a.ids[row * top + j];
            t = load_as_f32<DT>(a.teacher, row * top + j);
        }
        if (id >= V) bad = true;
        if (id < 0 || id >= V || t == -INFINITY) {
            id = -1;
            t = -INFINITY;
        }
        if constexpr (PART == DISTILL_STATS) {
            a.list[row * top + j] = id >= 0 ? load_as_f32<DT>(a.logits, base + id) : 0.0f;
        } else {
            s_id[j] = id;
            s_t[j] = t;
            s_z[j] = PART == DISTILL_GRAD ? a.list[row * top + j]
                     : id >= 0            ? load_as_f32<DT>(a.logits, base + id)
                                          : 0.0f;
        }
    }

    // ---- maximum and sum of exponentials ----
    float m = zedge, s = edge >= 0 && zedge != -INFINITY ? 1.0f : 0.0f;
    if constexpr (PART != DISTILL_GRAD) {
        if (zedge != zedge) s = zedge;          // (a maximum passes over NaN)
        auto add = [&](const float (&z)[VEC], float b) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) s += exp2_fast((z[e] - b) * a.c);
        };
        {
            const float m0 = m;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (v0 + tid + i * THREADS < v1) {
                    float z[VEC];
                    unpack<DT>(held[i], z);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) m = fmaxf(m, z[e]);
                }
            const float b = m == -INFINITY ? 0.0f : m;
            s *= exp2_fast((m0 - b) * a.c);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (v0 + tid + i * THREADS < v1) {
                    float z[VEC];
                    unpack<DT>(held[i], z);
                    add(z, b);
                }
        }
#pragma unroll 4
        for (int v = v0 + tid + NV * THREADS; v < v1; v += THREADS) {
            float z[VEC];
            unpack<DT>(body[v], z);
            float vm = z[0];
#pragma unroll
            for (int e = 1; e < VEC; ++e) vm = fmaxf(vm, z[e]);
            if (vm > m) {
                s *= exp2_fast((m - vm) * a.c);
                m = vm;
            }
            add(z, m == -INFINITY ? 0.0f : m);
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), a.c);
        if (lane == 0) {
            s_m[wave] = m;
            s_s[wave] = s;
        }
        bad = __syncthreads_or(bad);
        m = s_m[0];
        s = s_s[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) merge(m, s, s_m[w], s_s[w], a.c);
    }
    if constexpr (PART == DISTILL_STATS) {
        if (tid == 0) a.part[row * a.segs + seg] = make_float2(m, s);
        return;
    }
    if constexpr (PART == DISTILL_GRAD) {
        // (every wave joins the row's segments, at most a wave's lanes)
        const float2 p = lane < a.segs ? a.part[row * a.segs + lane] : make_float2(-INFINITY, 0.0f);
        m = p.x;
        s = p.y;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) merge(m, s, __shfl_xor(m, o), __shfl_xor(s, o), a.c);
        bad = __syncthreads_or(bad);
    }
    // log2 of a token's probability; the maximum leaves first, while the difference is exact or small
    const float ls = bad ? NAN : __builtin_amdgcn_logf(s);
    auto log2q = [&](float z) { return __builtin_fmaf(z - m, a.c, -ls); };

    // ---- the teacher's distribution over its list (every wave computes its sums) ----
    float tm = -INFINITY, ts = 0.0f;
    bool nan_t = false;
    for (int j = lane; j < top; j += 64) {
        tm = fmaxf(tm, s_t[j]);
        nan_t |= s_t[j] != s_t[j];
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) tm = fmaxf(tm, __shfl_xor(tm, o));
    const bool counts = tm != -INFINITY || __any(nan_t) || bad;
    const float tb = tm == -INFINITY ? 0.0f : tm;
    for (int j = lane; j < top; j += 64) ts += exp2_fast((s_t[j] - tb) * a.c);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) ts += __shfl_xor(ts, o);
    const float tl = __builtin_amdgcn_logf(ts);

    // ---- the gradient but for the listed tokens ----
    const float g = counts ? a.T * dloss : 0.0f;
    u32x4* out = reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.grad) + (base + head) * (16 / VEC));
    auto value = [&](float z) { return counts ? g * exp2_fast(log2q(z)) : 0.0f; };
    if (a.grad) {
        auto write = [&](int v, const u32x4& raw) {
            float z[VEC];
            unpack<DT>(raw, z);
#pragma unroll
            for (int e = 0; e < VEC; ++e) z[e] = value(z[e]);
            __builtin_nontemporal_store(pack<DT>(z), &out[v]);
        };
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (v0 + tid + i * THREADS < v1) write(v0 + tid + i * THREADS, held[i]);
#pragma unroll 4
        for (int v = v0 + tid + NV * THREADS; v < v1; v += THREADS) write(v, body[v]);
        if (edge >= 0) store_as<DT>(a.grad, base + edge, value(zedge));
    }

    // ---- loss, and the listed tokens' gradient ----
    auto log2p = [&](int j) { return (s_t[j] - tb) * a.c - tl; };
    if (first && wave == 0) {
        // T (log p - log q) = (t - tb) + (m - z) + T ln 2 (ls - tl): the logits enter as they are (times log2(e) / T, a
        // logit at its type's lowest value would pass fp32), and their differences are exact or small
        const float base = a.T * kLn2 * (ls - tl);
        float l = 0.0f;
        for (int j = lane; j < top; j += 64) {
            const float p = exp2_fast(log2p(j));
            if (p > 0.0f || p != p) l += p * ((s_t[j] - tb) + (m - s_z[j]) + base);
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) l += __shfl_xor(l, o);
        if (bad) l = NAN;
        if (lane == 0) a.loss[row] = counts ? a.T * l : 0.0f;
    }
    if (!a.grad || !counts) return;
    // other threads wrote the listed tokens' values: every store has to be done before they are written again
    wait_vmcnt<0>();
    __syncthreads();
#pragma unroll 1
    for (int j = tid; j < top; j += THREADS) {
        const int32_t id = s_id[j];
        if (id < 0) continue;
        if (PART == DISTILL_GRAD) {         // another segment's?
            const int v = (id - head) / VEC;
            if (id < head || id >= tail0 ? !first : v < v0 || v >= v1) continue;
        }
        // a token's first entry carries the mass of all of its entries
        float p = 0.0f;
        bool own = true;
#pragma unroll 4
        for (int i = 0; i < top; ++i)
            if (s_id[i] == id) {
                own &= i >= j;
                p += exp2_fast(log2p(i));
            }
        if (own) store_as<DT>(a.grad, base + id, g * (exp2_fast(log2q(s_z[j])) - p));
    }
}

// (a launch holds fewer than 2^32 threads)
constexpr int64_t kMaxRowBlocks = 1 << 20;
template <int DT, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS, 4) distill_kernel(DistillArgs a) {
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        distill_row<DT, THREADS, NV, DISTILL_ROW>(a, row, 0);
        __syncthreads();
    }
}

// Few long rows, in segments: a launch for the statistics, and one that joins them and writes the gradient.  One
// workgroup a row is bound by what a compute unit loads and exponentiates.
constexpr int kMaxSegments = 1024, kMaxSegmentRows = 192;
template <int DT, DistillPart PART>
__global__ void __launch_bounds__(256, 4) distill_segment_kernel(DistillArgs a) {
    const int row = (int)blockIdx.y;
    distill_row<DT, 256, 4, PART>(a, row, (int)blockIdx.x);
}

template <int DT>
hipError_t launch_distill_segments(const DistillArgs& a, hipStream_t st) {
    distill_segment_kernel<DT, DISTILL_STATS><<<dim3((unsigned)a.segs, (unsigned)a.n), 256, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    distill_segment_kernel<DT, DISTILL_GRAD><<<dim3(a.grad ? (unsigned)a.segs : 1u, (unsigned)a.n), 256, 0, st>>>(a);
    return hipGetLastError();
}

template <int DT, int THREADS, int NV>
hipError_t launch_distill(const DistillArgs& a, hipStream_t st) {
    distill_kernel<DT, THREADS, NV><<<(unsigned)std::min(a.n, kMaxRowBlocks), THREADS, 0, st>>>(a);
    return hipGetLastError();
}

// ---- cross entropy ----

struct RowState {          // arrays of n tokens each
    const int64_t* targets;
    const float* dloss;
    float* zt;             // the target's logit
    float* top;            // the largest logit
    float* ls;             // log2 of the sum of exponentials above it
    float* w;              // row weight of the gradient, 0 for a token that does not count
    float* loss;
    float* own;            // each token's entry of the logits' gradient at its target
    float* peak;           // the largest of them
};

// D rows are vocabulary rows, D columns tokens: a lane's values all belong to
// one token, so a tile's maximum and sum are reductions over registers.  4096 x
// 4096 x 131072 bf16: 3.38 ms, 1.30 PFLOP/s, bound by the products; 2048 x 1024
// x 50021: 0.24 ms, 0.88 (16 chunks a tile, an exponential for every 1024 of K).
template <int WM, int WN, int AM, int AN>
struct StatsEpilogue {
    float2* part;          // [tiles_m][n]
    RowState rs;
    __device__ void operator()(const floatx16 (&acc)[AM][AN], int tm, int, int m0, int n0, int M, int N,
                               uint8_t* lds) const {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int wm = wave / WN, wn = wave - wm * WN, l32 = lane & 31, hi = lane >> 5;
        float2* red = reinterpret_cast<float2*>(lds);            // [WM][BN]
        constexpr int BN = WN * AN * 32;
        __syncthreads();                                         // the last chunk is read
        if (m0 == 0 && n0 == 0 && tid == 0) *rs.peak = 0.0f;
        const int v0 = m0 + wm * AM * 32 + 4 * hi;               // vocabulary row of register 0
        const bool edge = m0 + WM * AM * 32 > M;
#pragma unroll
        for (int b = 0; b < AN; ++b) {
            const int col = wn * AN * 32 + b * 32 + l32;
            const int t = n0 + col;
            // the target as a row of this lane's first register
            const int64_t tv = t < N ? rs.targets[t] : -1;
            const int target = tv >= 0 && tv < M ? (int)tv - v0 : -1;
            // (rarely does a wave's part of the vocabulary hold any of its tokens' targets)
            if (__any(target >= 0 && target < AM * 32)) {
                float z = 0.0f;
                bool mine = false;
#pragma unroll
                for (int a = 0; a < AM; ++a)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (a * 32 + gemm_row(r, 0) == target) {
                            z = acc[a][b][r];
                            mine = true;
                        }
                if (mine) rs.zt[t] = z;
            }
            float m = -INFINITY, s = 0.0f;
            auto reduce = [&](auto last_tile) {
                constexpr bool kEdge = decltype(last_tile)::value;
#pragma unroll
                for (int a = 0; a < AM; ++a)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (!kEdge || v0 + a * 32 + gemm_row(r, 0) < M) m = fmaxf(m, acc[a][b][r]);
                const float bm = m == -INFINITY ? 0.0f : m;
#pragma unroll
                for (int a = 0; a < AM; ++a)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float e = exp2_fast((acc[a][b][r] - bm) * kLog2e);
                        if (!kEdge || v0 + a * 32 + gemm_row(r, 0) < M) s += e;
                    }
            };
            if (edge) reduce(std::true_type{});
            else reduce(std::false_type{});
            merge(m, s, __shfl_xor(m, 32), __shfl_xor(s, 32), kLog2e);
            if (hi == 0) red[wm * BN + col] = make_float2(m, s);
        }
        __syncthreads();
        for (int col = tid; col < BN; col += GemmTile<WM, WN, AM, AN>::kThreads) {
            if (n0 + col >= N) continue;
            float2 v = red[col];
#pragma unroll
            for (int w = 1; w < WM; ++w) merge(v.x, v.y, red[w * BN + col].x, red[w * BN + col].y, kLog2e);
            part[(int64_t)tm * N + n0 + col] = v;
        }
    }
};

__device__ __forceinline__ float row_weight(const RowState& rs, int64_t t) {
    return rs.targets[t] < 0 ? 0.0f : rs.dloss ? rs.dloss[t] : 1.0f;
}

// dloss (P - 1 at the target) of a piece of the vocabulary, in 16 bits, as
// [row][token].  Tokens up to a multiple of 8 and rows up to the tile's end are
// written (zeros past the ends): the products that read them walk whole 16-byte
// groups.  Neighbouring lanes hold neighbouring tokens: each pair of lanes swaps
// half of its values, so that every store carries two tokens of a row.  4096 x
// 4096 x 131072 bf16: 3.67 ms, 1.20 PFLOP/s, products, exponentials and stores.
enum GradScale {
    GRAD_CALL = 1,         // scaled by the call's peak
    GRAD_OWN = 2,          // by each token's own
    GRAD_BOTH = 3
};
template <int DT, int SCALE, int WM, int WN, int AM, int AN>
struct GradEpilogue {
    uint16_t* dlt;         // [piece][np] (GRAD_CALL)
    uint16_t* dlx;         // and by tokens (GRAD_OWN)
    int piece, np;
    int64_t v0;            // first vocabulary row of the piece
    RowState rs;
    __device__ void operator()(const floatx16 (&acc)[AM][AN], int, int, int m0, int n0, int M, int N, uint8_t*) const {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        const int wm = wave / WN, wn = wave - wm * WN, l32 = lane & 31, hi = lane >> 5;
        const float scale = SCALE & GRAD_CALL ? grad_scale(*rs.peak) : 1.0f;
        const bool odd = lane & 1;
        // the tile's rows from its corner: at most 255 pitches of kMaxPitch
        const __amdgpu_buffer_rsrc_t ro = buffer_rsrc(dlt + (int64_t)m0 * np + n0, kOutOfRange);
        const __amdgpu_buffer_rsrc_t rx = buffer_rsrc(dlx + (int64_t)m0 * np + n0, kOutOfRange);
#pragma unroll
        for (int b = 0; b < AN; ++b) {
            const int col = wn * AN * 32 + b * 32 + l32, t = n0 + col;
            const int64_t tv = t < N ? rs.targets[t] - v0 : -1;
            const int target = tv >= 0 && tv < M ? (int)tv - m0 : -1;
            const float top = t < N ? rs.top[t] : 0.0f, ls = t < N ? rs.ls[t] : 0.0f;
            const float w0 = t < N ? rs.w[t] : 0.0f, wc = w0 * scale;
            const float wo = SCALE & GRAD_OWN ? w0 * (t < N ? grad_scale(rs.own[t]) : 1.0f) : 0.0f;
            const uint32_t live = w0 != 0.0f ? 0xffffu : 0u;           // (zeros whatever the logits are)
#pragma unroll
            for (int a = 0; a < AM; ++a)
#pragma unroll
                for (int r = 0; r < 16; r += 2) {
                    const int v = (wm * AM + a) * 32 + gemm_row(r, hi);        // rows v and v + 1
                    float p[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        p[e] = exp2_fast(__builtin_fmaf(acc[a][b][r + e] - top, kLog2e, -ls));
                        if (v + e == target) p[e] -= 1.0f;
                    }
                    // even lanes keep row v of both tokens, odd lanes row v + 1
                    const int row = v + (odd ? 1 : 0);
                    const bool in = (t & ~1) < np && m0 + row < piece;
                    const uint32_t off = in ? (uint32_t)(row * np + (col & ~1)) * 2u : kOutOfRange;
                    auto put = [&](__amdgpu_buffer_rsrc_t to, float w) {
                        uint32_t o[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) o[e] = f32_to_tile<DT>(m0 + v + e < M ? p[e] * w : 0.0f) & live;
                        const uint32_t got = (uint32_t)__builtin_amdgcn_mov_dpp((int)(odd ? o[0] : o[1]), 0xB1, 0xF, 0xF, true);
                        const uint32_t two = odd ? got | o[1] << 16 : o[0] | got << 16;
                        __builtin_amdgcn_raw_buffer_store_b32(two, to, off, 0, 0);
                    };
                    if constexpr ((SCALE & GRAD_CALL) != 0) put(ro, wc);
                    if constexpr ((SCALE & GRAD_OWN) != 0) put(rx, wo);
                }
        }
    }
};

// dst[c][r] = src[r][c] for r < R, zero for R <= r < pitch and for rows that do not count.
struct Transpose {
    const uint16_t* src;
    uint16_t* dst;
    int R, C, pitch;       // C the source's pitch, a multiple of 8, as pitch is
    int tiles_r, tiles;    // 64 x 64 tiles along r, in all (0: nothing to do)
};

__device__ __forceinline__ void transpose_tile(const Transpose& a, int tile_id, const RowState& rows) {
    __shared__ __attribute__((aligned(16))) uint16_t tile[64][72];
    const int r0 = tile_id % a.tiles_r * 64, c0 = tile_id / a.tiles_r * 64;
    const int tid = threadIdx.x;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = r0 + (tid >> 3) + 32 * j, c = c0 + 8 * (tid & 7);
        u32x4 v{0, 0, 0, 0};
        if (r < a.R && c < a.C && row_weight(rows, r) != 0.0f)
            v = *reinterpret_cast<const u32x4*>(a.src + (int64_t)r * a.C + c);
        *reinterpret_cast<u32x4*>(&tile[(tid >> 3) + 32 * j][8 * (tid & 7)]) = v;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = c0 + (tid >> 3) + 32 * j, r = r0 + 8 * (tid & 7);
        if (c >= a.C || r >= a.pitch) continue;
        uint16_t o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = tile[8 * (tid & 7) + e][(tid >> 3) + 32 * j];
        u32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = o[2 * e] | (uint32_t)o[2 * e + 1] << 16;
        *reinterpret_cast<u32x4*>(a.dst + (int64_t)c * a.pitch + r) = v;
    }
}

// Maximum, sum, loss and row weight of every token from its tiles' parts: TOK
// tokens a workgroup, 256 / TOK threads a token (sixteen tokens make whole
// lines; four are sooner done where there are few).
template <int TOK>
__device__ __forceinline__ void join_tokens(const RowState& rs, const float2* part, int tiles, int n, int64_t V) {
    constexpr int kParts = 256 / TOK;
    __shared__ float2 red[kParts][TOK];
    const int tok = threadIdx.x % TOK, p = threadIdx.x / TOK;
    const int t = blockIdx.x * TOK + tok;
    float m = -INFINITY, s = 0.0f;
    if (t < n)
#pragma unroll 4
        for (int i = p; i < tiles; i += kParts) {
            const float2 v = part[(int64_t)i * n + t];
            merge(m, s, v.x, v.y, kLog2e);
        }
    red[p][tok] = make_float2(m, s);
    __syncthreads();
    if (p != 0) return;
    float peak = 0.0f;
    if (t < n) {
#pragma unroll 8
        for (int w = 1; w < kParts; ++w) merge(m, s, red[w][tok].x, red[w][tok].y, kLog2e);
        const int64_t target = rs.targets[t];
        float ls = __builtin_amdgcn_logf(s);
        const float w = row_weight(rs, t);
        float l = 0.0f;
        if (target >= V) {
            ls = l = NAN;
        } else if (target >= 0) {
            l = (m - rs.zt[t]) + kLn2 * ls;
            // (below 2^-20 of the weight the difference from 1 is rounding)
            const float v = fabsf(w) * fmaxf(1.0f - exp2_fast(__builtin_fmaf(rs.zt[t] - m, kLog2e, -ls)), 0x1p-20f);
            if (v < INFINITY) peak = v;
        }
        rs.loss[t] = l;
        rs.top[t] = m;
        rs.ls[t] = ls;
        rs.w[t] = w;
        rs.own[t] = peak;
    }
#pragma unroll
    for (int o = 1; o < TOK; o <<= 1) peak = fmaxf(peak, __shfl_xor(peak, o));
    // (bits of positive floats are in their order, and a maximum does not depend on the order of its arguments)
    if (tok == 0 && peak > 0.0f) atomicMax(reinterpret_cast<unsigned*>(rs.peak), __float_as_uint(peak));
}

// Between the statistics and the gradient, in one launch: the tokens' joins, and for dW the transposed inputs (rows
// that do not count left out: zeros times what they hold may not reach dW).
template <int TOK>
__global__ void __launch_bounds__(256) join_kernel(RowState rs, const float2* part, int tiles, int n, int64_t V,
                                                   Transpose x) {
    const int joins = (n + TOK - 1) / TOK, b = (int)blockIdx.x;
    if (b < joins) join_tokens<TOK>(rs, part, tiles, n, V);
    else transpose_tile(x, b - joins, rs);
}

template <int TOK>
hipError_t launch_join(const RowState& rs, const float2* part, int tiles, int n, int64_t V, const Transpose& x,
                       hipStream_t st) {
    const unsigned blocks = (unsigned)((n + TOK - 1) / TOK + x.tiles);
    join_kernel<TOK><<<blocks, 256, 0, st>>>(rs, part, tiles, n, V, x);
    return hipGetLastError();
}

int round_up(int64_t v, int to) { return (int)((v + to - 1) / to * to); }

}  // namespace

template <int DT, int SCALE>
static hipError_t launch_grad(const GemmOperands& g, uint16_t* dlt, uint16_t* dlx, int piece, int np, int64_t v0,
                              const RowState& rs, hipStream_t st) {
    const GemmPlan p = gemm_plan(g.M, g.N, g.K, 0);
    return p.big ? launch_gemm<DT, 2, 4, 4, 2, false>(g, p, GradEpilogue<DT, SCALE, 2, 4, 4, 2>{dlt, dlx, piece, np, v0, rs}, st)
                 : launch_gemm<DT, 2, 2, 2, 2, false>(g, p, GradEpilogue<DT, SCALE, 2, 2, 2, 2>{dlt, dlx, piece, np, v0, rs}, st);
}

template <int DT>
static hipError_t cross_entropy(aq_loss* L, const uint16_t* X, const uint16_t* W, const RowState& rs, uint16_t* dX,
                                uint16_t* dW, int n, hipStream_t st) {
    const int V = L->desc.vocab, F = L->desc.features, piece = L->piece, np = round_up(n, 8);
    hipError_t e;
    GemmOperands g{};
    g.zero = L->d_zero;
    g.A = W;
    g.lda = F;
    g.M = V;
    g.B = X;
    g.ldb = F;
    g.N = n;
    g.K = F;
    GemmPlan p = gemm_plan(V, n, F, 0);
    e = p.big ? launch_gemm<DT, 2, 4, 4, 2, false>(g, p, StatsEpilogue<2, 4, 4, 2>{L->d_part, rs}, st)
              : launch_gemm<DT, 2, 2, 2, 2, false>(g, p, StatsEpilogue<2, 2, 2, 2>{L->d_part, rs}, st);
    if (e != hipSuccess) return e;
    const int side = p.big ? 256 : 128;
    const int tiles_r = (np + 63) / 64;
    const Transpose tx = dW ? Transpose{X, L->d_xt, n, F, np, tiles_r, tiles_r * ((F + 63) / 64)} : Transpose{};
    e = n > 64 ? launch_join<16>(rs, L->d_part, (V + side - 1) / side, n, V, tx, st)
               : launch_join<4>(rs, L->d_part, (V + side - 1) / side, n, V, tx, st);
    if (e != hipSuccess || (!dX && !dW)) return e;
    const GemmPlan px = gemm_plan(n, F, std::min(V, piece), L->dx_bytes);
    const float* own = own_peaks(DT) ? rs.own : nullptr;
    uint16_t* dlx = own_peaks(DT) && dW ? L->d_dlx : L->d_dlt;       // dX's operand
    for (int64_t v0 = 0; v0 < V; v0 += piece) {
        const int rows = (int)std::min<int64_t>(piece, V - v0);
        const bool first = v0 == 0, last = v0 + piece >= V;
        g.A = W + v0 * F;
        g.M = rows;
        if constexpr (own_peaks(DT))
            e = !dW   ? launch_grad<DT, GRAD_OWN>(g, nullptr, dlx, piece, np, v0, rs, st)
                : !dX ? launch_grad<DT, GRAD_CALL>(g, L->d_dlt, nullptr, piece, np, v0, rs, st)
                      : launch_grad<DT, GRAD_BOTH>(g, L->d_dlt, dlx, piece, np, v0, rs, st);
        else e = launch_grad<DT, GRAD_CALL>(g, L->d_dlt, nullptr, piece, np, v0, rs, st);
        if (e != hipSuccess) return e;
        if (dX) {
            // the sum runs over rows of both operands; dX adds up over the pieces, and over the splits of each
            GemmOperands d = g;
            d.A = dlx;
            d.lda = np;
            d.M = n;
            d.B = W + v0 * F;
            d.N = F;
            d.K = rows;
            const bool whole = px.splits == 1 && last;
            const StoreArgs<DT> s{dX, L->d_dx, F, rs.peak, own};
            e = whole ? (first ? launch_store_gemm<DT, true, STORE_OUT>(d, px, s, st)
                               : launch_store_gemm<DT, true, STORE_LAST>(d, px, s, st))
                      : (first ? launch_store_gemm<DT, true, STORE_SUM>(d, px, s, st)
                               : launch_store_gemm<DT, true, STORE_ADD>(d, px, s, st));
            if (e == hipSuccess && last && !whole)
                e = launch_split_sum<DT, own_peaks(DT)>(L->d_dx, px.splits, n, F, dX, F, rs.peak, own, st);
            if (e != hipSuccess) return e;
        }
        if (dW) {
            GemmOperands d = g;
            d.A = L->d_dlt;
            d.B = L->d_xt;
            d.lda = d.ldb = np;
            d.M = rows;
            d.N = F;
            d.K = np;
            e = launch_store_gemm<DT, false, STORE_OUT>(d, gemm_plan(rows, F, np, 0),
                                                        StoreArgs<DT>{dW + v0 * F, nullptr, F, rs.peak, nullptr}, st);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

// Rows in segments: as many as leave half of the compute units without one, of 32768 values and more (what a workgroup
// exponentiates bounds it, so values count, not bytes), and up to three quarters of that many, three times as long.  us,
// whole rows / segments, fp32 and bf16:
//   1 row    24579 values  9.4 / 9.4, 10.5 / 9.6    32771 10.7 / 10.0, 11.5 / 9.3      131075 30.5 / 9.2, 27.4 / 9.4
//   64 rows  24579        11.1 / 11.5, 11.4 / 11.4  32771 13.1 / 11.7, 12.4 / 11.6     131075 32.7 / 19.8, 28.6 / 14.3
//   128      24579        11.8 / 12.7, 12.0 / 12.3  32771 13.9 / 13.6, 12.7 / 12.3     131075 53.7 / 39.2, 29.2 / 21.3
//   160      65539        24.2 / 26.1, 19.7 / 17.3  98307 42.6 / 37.7, 24.1 / 21.0     131075 55.7 / 47.1, 30.7 / 27.9
//   200      65539        31.9 / 32.3, 19.9 / 19.7  98307 45.7 / 45.6, 24.7 / 26.4     131075 59.4 / 56.2, 36.2 / 34.0
//   256      65539        35.9 / 39.6, 20.2 / 21.8  98307 52.5 / 53.5, 28.9 / 32.6     131075 67.5 / 67.9, 39.2 / 41.3
static bool distill_segmented(int64_t n, int64_t V) { return n <= 128 ? V >= 32768 : n <= kMaxSegmentRows && V >= 98304; }

template <int DT>
static hipError_t distill(DistillArgs a, hipStream_t st) {
    const int64_t vecs = a.V / Store<DT>::kVec;
    if (distill_segmented(a.n, a.V)) {
        a.segs = (int)std::min<int64_t>(64, kMaxSegments / a.n);
        a.seg_vecs = (int)((vecs + a.segs - 1) / a.segs);
        return launch_distill_segments<DT>(a, st);
    }
    // More rows than the 512 that larger workgroups hold at a time (two a compute unit) go to smaller ones (four), up to
    // the length where reading again what those do not hold costs more: us, smaller / larger, 4096 rows of 96, 108, 112
    // and 128 KB, bf16 169 / 177, 187 / 193, 203 / 200, 250 / 224, fp16 164 / 175, 184 / 193, 199 / 199, 246 / 222; fp32,
    // 48, 60, 64 and 68 KB, 82 / 91, 102 / 103, 115 / 114, 116 / 112.  1024 rows, 64 KB, bf16 29.9 / 33.6; 600, 92 KB,
    // 32.8 / 32.9; 512, 64 KB, 19.6 / 18.2.
    return a.n > 512 && vecs <= (DT == AQ_F32 ? 4096 : 7168) ? launch_distill<DT, 256, 16>(a, st)
                                                             : launch_distill<DT, 512, 14>(a, st);
}

}  // namespace aq

namespace {

void free_loss(aq_loss* L) {
    void* ptrs[] = {L->d_seg, L->d_list, L->d_zero, L->d_part, L->d_row, L->d_dlt, L->d_dlx, L->d_xt, L->d_dx};
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

constexpr size_t kSplitBytes = size_t(64) << 20;   // most that a K split's sums of dX take

// The gradients' workspace (the first call that asks for one allocates it).
aq_status grad_workspace(aq_loss* L, bool dx, bool dw, void* stream) {
    // (from the call on that makes it both gradients' handle, whether or not one call asks for both)
    const bool two = (dx || L->d_dx) && (dw || L->d_xt) && aq::own_peaks(L->desc.dtype);
    if (L->d_dlt && (!dx || L->d_dx) && (!dw || L->d_xt) && (!two || L->d_dlx)) return AQ_OK;
    if (aq::capturing(static_cast<hipStream_t>(stream)))
        return api_fail(AQ_ERR_UNSUPPORTED, "the first call with a gradient allocates: not under graph capture");
    const size_t n = (size_t)(L->desc.max_tokens + 7) / 8 * 8, F = (size_t)L->desc.features, P = (size_t)L->piece;
    aq_status s = AQ_OK;
    s = alloc(&L->d_dlt, n * P * 2, "gradient workspace");
    if (s == AQ_OK && two) s = alloc(&L->d_dlx, n * P * 2, "gradient workspace");
    if (s == AQ_OK && dx && !L->d_dx) {
        const int64_t mt = L->desc.max_tokens;
        const size_t split = aq::gemm_split_bytes(mt, F, std::min<int64_t>(L->desc.vocab, L->piece), kSplitBytes);
        const size_t bytes = std::max(split, L->piece < L->desc.vocab ? (size_t)mt * F * 4 : (size_t)16);
        s = alloc(&L->d_dx, bytes, "gradient workspace");
        if (s == AQ_OK) L->dx_bytes = bytes;
    }
    if (s == AQ_OK && dw) s = alloc(&L->d_xt, n * F * 2, "gradient workspace");
    return s;
}

// A loss is written while other workgroups still read dloss (joined rows of the cross entropy, segments of the
// distillation; a whole row's own workgroup alone reads its dloss, and before it writes its loss).
bool overlaps(const float* a, const float* b, int64_t n) { return a && b && a < b + n && b < a + n; }

bool misaligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

aq_status check_call(const aq_loss* L, int64_t n) {
    if (n < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "n must be >= 1");
    if (n > L->desc.max_tokens) return api_fail(AQ_ERR_INVALID_ARGUMENT, "tokens exceed max_tokens");
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return api_hip_fail(e, "hipGetDevice");
    if (dev != L->device) return api_fail(AQ_ERR_INVALID_ARGUMENT, "the losses were created on another device");
    return AQ_OK;
}

}  // namespace

extern "C" {

aq_status aq_loss_create(const aq_loss_desc* desc, aq_loss** out) {
    if (out) *out = nullptr;
    if (!desc || !out) return api_fail(AQ_ERR_INVALID_ARGUMENT, "null pointer argument");
    if (desc->vocab < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "vocab must be >= 1");
    if (desc->vocab > (1 << 30)) return api_fail(AQ_ERR_UNSUPPORTED, "vocab above 2^30");
    if (desc->features < 0) return api_fail(AQ_ERR_INVALID_ARGUMENT, "features must be >= 0");
    if (desc->dtype != AQ_F32 && desc->dtype != AQ_F16 && desc->dtype != AQ_BF16)
        return api_fail(AQ_ERR_INVALID_ARGUMENT, "dtype must be F32, F16 or BF16");
    if (desc->max_tokens < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "max_tokens must be >= 1");
    if (desc->max_tokens > (1 << 24)) return api_fail(AQ_ERR_UNSUPPORTED, "max_tokens above 2^24");
    if (desc->features && desc->dtype == AQ_F32)
        return api_fail(AQ_ERR_UNSUPPORTED, "the cross entropy takes fp16 or bf16 inputs and head weights");
    if (desc->features % 8 != 0) return api_fail(AQ_ERR_UNSUPPORTED, "features must be a multiple of 8");
    if (desc->features > aq::kMaxPitch || (desc->features && desc->max_tokens > aq::kMaxPitch))
        return api_fail(AQ_ERR_UNSUPPORTED, "features, or max_tokens of a cross entropy, above 2^21");
    int ndev = 0;
    hipError_t e = hipGetDeviceCount(&ndev);
    if (e != hipSuccess || ndev < 1) return api_fail(AQ_ERR_DEVICE, "no HIP device available");
    aq_loss* L = new (std::nothrow) aq_loss();
    if (!L) return api_fail(AQ_ERR_OUT_OF_MEMORY, "host allocation");
    L->desc = *desc;
    e = hipGetDevice(&L->device);
    if (e != hipSuccess) {
        delete L;
        return api_hip_fail(e, "hipGetDevice");
    }
    const size_t few = (size_t)std::min<int64_t>(desc->max_tokens, aq::kMaxSegmentRows);
    aq_status s = alloc(&L->d_seg, aq::kMaxSegments * sizeof(float2), "segment statistics");
    if (s == AQ_OK) s = alloc(&L->d_list, few * aq::kMaxTop * sizeof(float), "listed logits");
    if (s == AQ_OK && desc->features) {
        // a piece's gradient takes at most 128 MiB, its head rows too
        const int64_t most = std::min(aq::kMaxPitch, std::max<int64_t>(256, (int64_t(64) << 20) / std::max<int64_t>(
                                                                              desc->max_tokens, desc->features)));
        const int64_t pieces = (desc->vocab + most - 1) / most;
        L->piece = (int)(((desc->vocab + pieces - 1) / pieces + 255) / 256 * 256);
        const size_t n = (size_t)desc->max_tokens, tiles = (size_t)(desc->vocab + 127) / 128;
        s = alloc(&L->d_zero, 256, "zero block");
        if (s == AQ_OK) s = alloc(&L->d_part, tiles * n * sizeof(float2), "row statistics");
        if (s == AQ_OK) s = alloc(&L->d_row, (5 * n + 1) * sizeof(float), "row state");
        if (s == AQ_OK && (e = hipMemset(L->d_zero, 0, 256)) != hipSuccess) s = api_hip_fail(e, "zero block");
        if (s == AQ_OK && (e = hipDeviceSynchronize()) != hipSuccess) s = api_hip_fail(e, "zero block");
    }
    if (s != AQ_OK) {
        free_loss(L);
        return s;
    }
    *out = L;
    return AQ_OK;
}

aq_status aq_loss_cross_entropy(aq_loss* L, const void* X, const void* W, const int64_t* targets, const float* dloss,
                                float* loss, void* dX, void* dW, int64_t n, void* stream) {
    if (!L || !X || !W || !targets || !loss) return api_fail(AQ_ERR_INVALID_ARGUMENT, "null pointer argument");
    if (!L->desc.features) return api_fail(AQ_ERR_INVALID_ARGUMENT, "created without features: distillation only");
    if (misaligned(X, 16) || misaligned(W, 16) || misaligned(dX, 16) || misaligned(dW, 16))
        return api_fail(AQ_ERR_INVALID_ARGUMENT, "X, W, dX and dW must be 16-byte aligned");
    if (misaligned(targets, 8)) return api_fail(AQ_ERR_INVALID_ARGUMENT, "targets must be 8-byte aligned");
    if (misaligned(dloss, 4) || misaligned(loss, 4))
        return api_fail(AQ_ERR_INVALID_ARGUMENT, "dloss and loss must be 4-byte aligned");
    aq_status s = check_call(L, n);
    if (s != AQ_OK) return s;
    if (overlaps(loss, dloss, n)) return api_fail(AQ_ERR_INVALID_ARGUMENT, "loss overlaps dloss");
    const int64_t F = L->desc.features, tiles_n = (n + 127) / 128;
    if (tiles_n * ((L->desc.vocab + 127) / 128) > aq::kMaxTiles || tiles_n * ((F + 127) / 128) > aq::kMaxTiles)
        return api_fail(AQ_ERR_UNSUPPORTED, "too many tokens times vocabulary or features for one call");
    if (dW && ((n + 63) / 64 * ((F + 63) / 64) + n / 4 + 2 >= (1 << 24)))    // the joining launch's workgroups
        return api_fail(AQ_ERR_UNSUPPORTED, "too many tokens times features for one call");
    if (dX || dW) {
        s = grad_workspace(L, dX != nullptr, dW != nullptr, stream);
        if (s != AQ_OK) return s;
    }
    const int64_t mt = L->desc.max_tokens;
    const aq::RowState rs{targets, dloss, L->d_row, L->d_row + mt, L->d_row + 2 * mt, L->d_row + 3 * mt, loss,
                          L->d_row + 4 * mt, L->d_row + 5 * mt};
    const auto st = static_cast<hipStream_t>(stream);
    const auto x = static_cast<const uint16_t*>(X), w = static_cast<const uint16_t*>(W);
    const auto dx = static_cast<uint16_t*>(dX), dw = static_cast<uint16_t*>(dW);
    const hipError_t e = L->desc.dtype == AQ_F16 ? aq::cross_entropy<AQ_F16>(L, x, w, rs, dx, dw, (int)n, st)
                                                 : aq::cross_entropy<AQ_BF16>(L, x, w, rs, dx, dw, (int)n, st);
    return e == hipSuccess ? AQ_OK : api_hip_fail(e, "cross entropy launch");
}

aq_status aq_loss_distill(aq_loss* L, const void* logits, const int32_t* ids, const void* teacher, int32_t top,
                          float temperature, const float* dloss, float* loss, void* dlogits, int64_t n, void* stream) {
    if (!L || !logits || !ids || !teacher || !loss) return api_fail(AQ_ERR_INVALID_ARGUMENT, "null pointer argument");
    if (top < 1) return api_fail(AQ_ERR_INVALID_ARGUMENT, "top must be >= 1");
    if (top > aq::kMaxTop) return api_fail(AQ_ERR_UNSUPPORTED, "top above 1024");
    if (!(temperature > 0.0f) || !std::isfinite(temperature))
        return api_fail(AQ_ERR_INVALID_ARGUMENT, "temperature must be positive and finite");
    if (!std::isfinite(aq::kLog2e / temperature)) return api_fail(AQ_ERR_UNSUPPORTED, "temperature below 2^-127");
    const unsigned b = L->desc.dtype == AQ_F32 ? 4 : 2;
    if (misaligned(logits, 16) || misaligned(dlogits, 16))
        return api_fail(AQ_ERR_INVALID_ARGUMENT, "logits and dlogits must be 16-byte aligned");
    if (misaligned(ids, 4) || misaligned(teacher, b) || misaligned(dloss, 4) || misaligned(loss, 4))
        return api_fail(AQ_ERR_INVALID_ARGUMENT, "ids, teacher, dloss and loss must be aligned to their values");
    const aq_status s = check_call(L, n);
    if (s != AQ_OK) return s;
    if (overlaps(loss, dloss, n) &&
        (loss != dloss || aq::distill_segmented(n, L->desc.vocab)))
        return api_fail(AQ_ERR_INVALID_ARGUMENT, "loss overlaps dloss");
    const aq::DistillArgs a{logits, ids, teacher, dloss, loss, dlogits, n, L->desc.vocab, top, aq::kLog2e / temperature,
                            temperature, 0, 0, L->d_seg, L->d_list};
    const auto st = static_cast<hipStream_t>(stream);
    const hipError_t e = L->desc.dtype == AQ_F32   ? aq::distill<AQ_F32>(a, st)
                         : L->desc.dtype == AQ_F16 ? aq::distill<AQ_F16>(a, st)
                                                   : aq::distill<AQ_BF16>(a, st);
    return e == hipSuccess ? AQ_OK : api_hip_fail(e, "distillation launch");
}

aq_status aq_loss_destroy(aq_loss* L) {
    if (!L) return AQ_OK;
    const hipError_t e = hipDeviceSynchronize();
    free_loss(L);
    return e == hipSuccess ? AQ_OK : api_hip_fail(e, "destroy");
}

}  // extern "C"
