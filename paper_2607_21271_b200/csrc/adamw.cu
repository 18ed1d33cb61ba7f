// AdamW over many tensors in one launch, with states in 32 or in 8 bits, and the global gradient norm that may precede it.
//
// Everything here moves memory: per element a step reads the gradient, the two states and the parameter (or its float master) and
// writes all but the gradient, 30 bytes with float states (float gradient, 16-bit parameter with master) or 18 with 8-bit ones, for
// about 20 operations.  The unit of work is a chunk of 2048 elements of one tensor: eight warps, each one block of 256 elements, eight
// per lane, so that the block that shares a scale is a warp and its maximum one reduction.  The table of tensors and the
// tensor of every chunk lie in the workspace; a CTA looks up its next 32 chunks at once, so that its loads of data do not wait for one
// entry of the table after the other.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdlib>
#include <new>

#include "eql_internal.h"
#include "packed.cuh"
#include "ptx_sm100.cuh"

namespace eql {
namespace {

constexpr int kBlock = 256;                 // elements that share a scale: one warp's
constexpr int kAdamThreads = 256;
constexpr int kChunk = kBlock * (kAdamThreads / 32);
// CTAs resident together, by their registers.  (With float states, 10.6 million weights and the norm: two 67 us, three 73, four 73; with
// 8-bit ones, 134 million: two 478, three 467, four 473.)
constexpr int kNormCtasPerSm = 4;
constexpr int step_ctas_per_sm(int bits) { return bits == 8 ? 3 : 2; }
constexpr int kNormUnroll = 4;              // chunks of gradients that a warp has on their way
constexpr int kTable = 32;                  // tensors that a CTA looks up at a time
constexpr int kMaxNormCtas = 1024;
constexpr float kE4m3Max = 448.0f, kE5m2Max = 57344.0f, kE5m2Least = 0x1p-16f, kTiny = 0x1p-100f;

// One tensor, as the kernels see it.
struct Tensor {
    void* param;
    float* master;
    const void* grad;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t numel;
    int32_t first_chunk;
    int32_t param_dtype, grad_dtype;
    float weight_decay, lr_scale;
    int32_t unused;           // (whole pieces of eight bytes)
};

// The optimiser's own state, at the start of the workspace.
struct Control {
    int64_t step, skipped;
    float factor, norm;
    int32_t skip;
    unsigned step_ticket, norm_ticket;
};
static_assert(sizeof(Control) <= kWsAlign, "the control block has one slot of the workspace");

struct Layout {
    size_t partials, tensors, chunks, total;
    int64_t n_chunks;
};

// What a step has in every element's formula (host: rounded once from double).
struct Rates {
    float lr, beta1, one_minus_beta1, beta2, one_minus_beta2, eps;
    float one;                // 1: see adamw_kernel
    double log_beta1, log_beta2;
    const float* lr_device;
};

// A lane's eight elements are two runs of four, 128 elements apart, so that a warp's access is one run of 128 elements.
constexpr int kRun = 128;

// Four neighbouring elements as they lie in memory, SIZE bytes each, in the first words; fetched before any of them is looked at.
template <int SIZE>
__device__ __forceinline__ uint4 load_raw4(const void* from) {
    if (SIZE == 4) return __ldcs(static_cast<const uint4*>(from));
    if (SIZE == 2) { const uint2 w = __ldcs(static_cast<const uint2*>(from)); return make_uint4(w.x, w.y, 0u, 0u); }
    return make_uint4(__ldcs(static_cast<const uint32_t*>(from)), 0u, 0u, 0u);
}
template <int SIZE>
__device__ __forceinline__ void store_raw4(void* to, const uint4& u) {
    if (SIZE == 4) __stcs(static_cast<uint4*>(to), u);
    if (SIZE == 2) __stcs(static_cast<uint2*>(to), make_uint2(u.x, u.y));
    if (SIZE == 1) __stcs(static_cast<uint32_t*>(to), u.x);
}
// The same, as far as a tensor goes: `left` elements from there on, the others count as zero.
template <int SIZE>
__device__ __forceinline__ uint4 load_some4(const void* from, int left) {
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j >= left) break;
        uint32_t& word = (&u.x)[j * SIZE / 4];
        if (SIZE == 4) word = static_cast<const uint32_t*>(from)[j];
        if (SIZE == 2) word |= (uint32_t)static_cast<const uint16_t*>(from)[j] << (16 * (j & 1));
        if (SIZE == 1) word |= (uint32_t)static_cast<const uint8_t*>(from)[j] << (8 * j);
    }
    return u;
}
template <int SIZE>
__device__ __forceinline__ void store_some4(void* to, int left, const uint4& u) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j >= left) break;
        const uint32_t word = (&u.x)[j * SIZE / 4];
        if (SIZE == 4) static_cast<uint32_t*>(to)[j] = word;
        if (SIZE == 2) static_cast<uint16_t*>(to)[j] = (uint16_t)(word >> (16 * (j & 1)));
        if (SIZE == 1) static_cast<uint8_t*>(to)[j] = (uint8_t)(word >> (8 * j));
    }
}
__device__ __forceinline__ float2 widen_pair(uint32_t u, int dtype) {
    if (dtype == EQL_FP16) return __half22float2(*reinterpret_cast<const __half2*>(&u));
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
__device__ __forceinline__ void widen4(const uint4& u, int dtype, float2* f) {
    if (dtype == EQL_FP32) {
        f[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
        f[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
    } else {
        f[0] = widen_pair(u.x, dtype);
        f[1] = widen_pair(u.y, dtype);
    }
}
__device__ __forceinline__ uint32_t narrow_pair(float2 f, int dtype) {
    if (dtype == EQL_FP16) {
        const __half2 h = __floats2half2_rn(f.x, f.y);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 narrow4(const float2* f, int dtype) {
    if (dtype == EQL_FP32) return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    return make_uint4(narrow_pair(f[0], dtype), narrow_pair(f[1], dtype), 0u, 0u);
}

template <__nv_fp8_interpretation_t KIND>
__device__ __forceinline__ float2 decode_pair(uint32_t codes, float2 scale) {
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, KIND);
    return mul2(__half22float2(__half2(r)), scale);
}
template <__nv_fp8_interpretation_t KIND>
__device__ __forceinline__ void decode4(uint32_t codes, float2 scale, float2* f) {
    f[0] = decode_pair<KIND>(codes & 0xffffu, scale);
    f[1] = decode_pair<KIND>(codes >> 16, scale);
}
template <__nv_fp8_interpretation_t KIND>
__device__ __forceinline__ uint32_t encode4(const float2* q) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(q[0], __NV_SATFINITE, KIND);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(q[1], __NV_SATFINITE, KIND);
    return lo | hi << 16;
}

// The largest of a warp's values, which are not negative: their bits are in the order of the values, NaN last.
__device__ __forceinline__ float warp_max(float v) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v))); }

// A CTA's chunks: all CTAs together sweep over the tensors, so that what is under way at a time lies close together in memory (with a
// contiguous run of chunks for each CTA, 134 million weights took 462 us instead of 389).  The tensors of the next chunks are looked up
// for all of them at once: use(table, first, count), entry i of the table being that of chunk first + i * gridDim.x.
template <typename Use>
__device__ __forceinline__ void for_chunks(char* ws, const Layout& lay, Tensor* table, Use&& use) {
    constexpr int kPieces = sizeof(Tensor) / 8;
    static_assert(sizeof(Tensor) % 8 == 0, "copied in pieces of eight bytes");
    const uint64_t* tensors = reinterpret_cast<const uint64_t*>(ws + lay.tensors);
    const int32_t* chunk_tensor = reinterpret_cast<const int32_t*>(ws + lay.chunks);
    for (int64_t first = blockIdx.x; first < lay.n_chunks; first += (int64_t)kTable * gridDim.x) {
        const int64_t left = (lay.n_chunks - first + gridDim.x - 1) / gridDim.x;
        const int count = left < kTable ? (int)left : kTable;
        __syncthreads();
        for (int i = threadIdx.x; i < count * kPieces; i += kAdamThreads) {
            const int entry = i / kPieces, piece = i - entry * kPieces;
            reinterpret_cast<uint64_t*>(table + entry)[piece] = tensors[(int64_t)chunk_tensor[first + (int64_t)entry * gridDim.x] * kPieces + piece];
        }
        __syncthreads();
        use(first, count);
    }
}
// The warp's block in chunk c: its first element, and how many its tensor has from there on (as far as a block goes).
struct Block {
    int64_t base;
    int count;
    __device__ __forceinline__ Block(const Tensor& x, int64_t c) : base((c - x.first_chunk) * kChunk + (threadIdx.x >> 5) * kBlock) {
        const int64_t left = x.numel - base;
        count = left >= kBlock ? kBlock : left > 0 ? (int)left : 0;
    }
};

// A lane's part of a block, as it lies in memory.
template <int BITS>
struct Fetched {
    uint4 g[2], p[2], m[2], v[2];
    float m_scale, v_scale;
};
// The same for the packed operations.
struct Formula {
    float2 factor, beta1, new1, beta2, new2, one, eps, root2;
};

// One block.  The moments are computed by separately rounded operations: in 8 bits, what lies next to the border of two codes goes by
// their last bit, and a plain program has to come to the same codes.  (The assembler makes one fused operation of a packed product
// and a packed sum, their rounding modes notwithstanding; a sum written as a * 1 + b, with a 1 that it does not know, is left alone.)
// The denominator may be a few float roundings off (approximate square root and reciprocal, about 2^-22): it moves the parameter by lr
// times that.
template <int BITS>
__device__ __forceinline__ void update(const Formula& f, Fetched<BITS>& b, int grad_dtype, int from_dtype, float2 keep, float2 size, float2* p) {
    float2 g[4], m[4], v[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        widen4(b.g[h], grad_dtype, g + 2 * h);
        widen4(b.p[h], from_dtype, p + 2 * h);
        if (BITS == 32) {
            widen4(b.m[h], EQL_FP32, m + 2 * h);
            widen4(b.v[h], EQL_FP32, v + 2 * h);
        } else {
            decode4<__NV_E4M3>(b.m[h].x, pair(b.m_scale), m + 2 * h);
            decode4<__NV_E5M2>(b.v[h].x, pair(b.v_scale), v + 2 * h);
        }
    }
    float most_m = 0.0f, most_v = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 gs = mul2(g[j], f.factor);
        m[j] = fma2(mul2(m[j], f.beta1), f.one, mul2(gs, f.new1));
        v[j] = fma2(mul2(v[j], f.beta2), f.one, mul2(mul2(gs, gs), f.new2));
        if (BITS == 8) {
            most_m = fmaxf(most_m, fmaxf(fabsf(m[j].x), fabsf(m[j].y)));
            most_v = fmaxf(most_v, fmaxf(v[j].x, v[j].y));
        }
        float2 root;
        asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root.x) : "f"(v[j].x));
        asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root.y) : "f"(v[j].y));
        p[j] = fma2(mul2(size, m[j]), reciprocal(fma2(root, f.root2, f.eps)), mul2(p[j], keep));
    }
    if (BITS == 32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            b.m[h] = narrow4(m + 2 * h, EQL_FP32);
            b.v[h] = narrow4(v + 2 * h, EQL_FP32);
        }
        return;
    }
    most_m = warp_max(most_m);
    most_v = warp_max(most_v);
    const bool fine_m = !(most_m < kTiny), fine_v = !(most_v < kTiny);
    // (To nearest: what a step moves by less than half of what lies between codes keeps its code.  That bounds beta2, see eqlinear.h.)
    // the block's four divisions, each in another lane: the inverse scales of m and v, and the scales
    const int lane = threadIdx.x & 31;
    const bool of_v = lane & 1, scale = lane & 2;
    const float most = of_v ? most_v : most_m, top = of_v ? kE5m2Max : kE4m3Max;
    const float ratio = (of_v ? fine_v : fine_m) ? __fdiv_rn(scale ? most : top, scale ? top : most) : 0.0f;
    const float2 im = pair(__shfl_sync(0xffffffffu, ratio, 0)), iv = pair(__shfl_sync(0xffffffffu, ratio, 1));
    float smallest = kE5m2Least;
    float2 qm[4], qv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        qm[j] = mul2(m[j], im);
        qv[j] = mul2(v[j], iv);
        smallest = fminf(smallest, fminf(qv[j].x, qv[j].y));
    }
    if (smallest < kE5m2Least && fine_v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (v[j].x > 0.0f) qv[j].x = fmaxf(qv[j].x, kE5m2Least);
            if (v[j].y > 0.0f) qv[j].y = fmaxf(qv[j].y, kE5m2Least);
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        b.m[h].x = encode4<__NV_E4M3>(qm + 2 * h);
        b.v[h].x = encode4<__NV_E5M2>(qv + 2 * h);
    }
    b.m_scale = b.v_scale = ratio;                            // lane 2's and lane 3's
}

// A block at a tensor's end.
template <int BITS>
__device__ __noinline__ void update_end(const Formula& f, const Tensor& x, int64_t base, int count, float2 keep, float2 size) {
    constexpr int S = BITS / 8;
    const int lane = threadIdx.x & 31;
    const int64_t block = base / kBlock;
    Fetched<BITS> b;
    float2 p[4];
    if (BITS == 8) { b.m_scale = x.m_scale[block]; b.v_scale = x.v_scale[block]; }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t at = base + h * kRun + lane * 4;
        const int left = count - h * kRun - lane * 4;
        b.g[h] = x.grad_dtype == EQL_FP32 ? load_some4<4>((const float*)x.grad + at, left) : load_some4<2>((const uint16_t*)x.grad + at, left);
        b.p[h] = x.master ? load_some4<4>(x.master + at, left) : x.param_dtype == EQL_FP32 ? load_some4<4>((const float*)x.param + at, left)
                                                                                          : load_some4<2>((const uint16_t*)x.param + at, left);
        b.m[h] = load_some4<S>((const char*)x.m + at * S, left);
        b.v[h] = load_some4<S>((const char*)x.v + at * S, left);
    }
    update<BITS>(f, b, x.grad_dtype, x.master ? (int)EQL_FP32 : x.param_dtype, keep, size, p);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t at = base + h * kRun + lane * 4;
        const int left = count - h * kRun - lane * 4;
        if (x.master) store_some4<4>(x.master + at, left, narrow4(p + 2 * h, EQL_FP32));
        if (x.param_dtype == EQL_FP32) store_some4<4>((float*)x.param + at, left, narrow4(p + 2 * h, EQL_FP32));
        else store_some4<2>((uint16_t*)x.param + at, left, narrow4(p + 2 * h, x.param_dtype));
        store_some4<S>((char*)x.m + at * S, left, b.m[h]);
        store_some4<S>((char*)x.v + at * S, left, b.v[h]);
    }
    if (BITS == 8 && lane == 2) x.m_scale[block] = b.m_scale;
    if (BITS == 8 && lane == 3) x.v_scale[block] = b.v_scale;
}

// GRAD, PARAM: the type that all tensors have there, or kMixed.
constexpr int kMixed = -1;
template <int BITS, int GRAD, int PARAM>
__global__ void __launch_bounds__(kAdamThreads, step_ctas_per_sm(BITS)) adamw_kernel(char* ws, Layout lay, Rates r) {
    constexpr int S = BITS / 8;
    ptx::grid_handover();
    Control* control = reinterpret_cast<Control*>(ws);
    __shared__ Tensor table[kTable];
    const int lane = threadIdx.x & 31;
    const int32_t skip = control->skip;
    if (!skip) {
        const double t = (double)(control->step + 1);
        const float lr = r.lr_device ? *r.lr_device : r.lr;
        const float correction1 = -expm1f((float)(t * r.log_beta1)), correction2 = -expm1f((float)(t * r.log_beta2));
        const Formula f{pair(control->factor), pair(r.beta1), pair(r.one_minus_beta1), pair(r.beta2), pair(r.one_minus_beta2), pair(r.one), pair(r.eps),
                        pair(rsqrtf(correction2))};
        // A block with 8-bit states is fetched while the one before is computed: its arithmetic takes as long as the memory does.
        constexpr bool kAhead = BITS == 8;
        for_chunks(ws, lay, table, [&](int64_t first, int count) {
            Fetched<BITS> next;
            bool fetched = false;
            auto fetch = [&](const Tensor& x, int64_t base) {
                const int64_t at = base + lane * 4;
                const int grad_dtype = GRAD == kMixed ? x.grad_dtype : GRAD, param_dtype = PARAM == kMixed ? x.param_dtype : PARAM;
                const char *m = (const char*)x.m + at * S, *v = (const char*)x.v + at * S;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    next.g[h] = grad_dtype == EQL_FP32 ? load_raw4<4>((const float*)x.grad + at + h * kRun) : load_raw4<2>((const uint16_t*)x.grad + at + h * kRun);
                    next.m[h] = load_raw4<S>(m + h * kRun * S);
                    next.v[h] = load_raw4<S>(v + h * kRun * S);
                }
                if (x.master) {
                    next.p[0] = load_raw4<4>(x.master + at);
                    next.p[1] = load_raw4<4>(x.master + at + kRun);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        next.p[h] = param_dtype == EQL_FP32 ? load_raw4<4>((const float*)x.param + at + h * kRun) : load_raw4<2>((const uint16_t*)x.param + at + h * kRun);
                }
                if (BITS == 8) { next.m_scale = x.m_scale[base / kBlock]; next.v_scale = x.v_scale[base / kBlock]; }
            };
            for (int i = 0; i < count; ++i) {
                const Tensor& x = table[i];
                const Block block(x, first + (int64_t)i * gridDim.x);
                const bool whole = block.count == kBlock;
                if (whole && !fetched) fetch(x, block.base);
                Fetched<BITS> now = next;
                fetched = false;
                if (kAhead && i + 1 < count) {
                    const Block after(table[i + 1], first + (int64_t)(i + 1) * gridDim.x);
                    fetched = after.count == kBlock;
                    if (fetched) fetch(table[i + 1], after.base);
                }
                if (block.count == 0) continue;
                const float rate = lr * x.lr_scale;
                const float2 keep = pair(1.0f - rate * x.weight_decay), size = pair(__fdividef(-rate, correction1));
                if (!whole) {
                    update_end<BITS>(f, x, block.base, block.count, keep, size);
                    continue;
                }
                const int grad_dtype = GRAD == kMixed ? x.grad_dtype : GRAD, param_dtype = PARAM == kMixed ? x.param_dtype : PARAM;
                float2 value[4];
                update<BITS>(f, now, grad_dtype, x.master ? (int)EQL_FP32 : param_dtype, keep, size, value);
                const int64_t at = block.base + lane * 4;
                if (x.master) {
                    store_raw4<4>(x.master + at, narrow4(value, EQL_FP32));
                    store_raw4<4>(x.master + at + kRun, narrow4(value + 2, EQL_FP32));
                }
                char *m = (char*)x.m + at * S, *v = (char*)x.v + at * S;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (param_dtype == EQL_FP32) store_raw4<4>((float*)x.param + at + h * kRun, narrow4(value + 2 * h, EQL_FP32));
                    else store_raw4<2>((uint16_t*)x.param + at + h * kRun, narrow4(value + 2 * h, param_dtype));
                    store_raw4<S>(m + h * kRun * S, now.m[h]);
                    store_raw4<S>(v + h * kRun * S, now.v[h]);
                }
                if (BITS == 8 && lane == 2) x.m_scale[block.base / kBlock] = now.m_scale;
                if (BITS == 8 && lane == 3) x.v_scale[block.base / kBlock] = now.v_scale;
            }
        });
    }
    // The last CTA to come here, when every CTA has read the control block, turns it to the next step.
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&control->step_ticket, 1u) == gridDim.x - 1) {
            if (skip) control->skipped += 1;
            else control->step += 1;
            control->factor = 1.0f;
            control->skip = 0;
            control->step_ticket = 0;
        }
    }
}

__device__ __forceinline__ double cta_sum(double v, double* shared) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < kAdamThreads / 32; ++w) s += shared[w];
    return s;
}

// Sum of squares in double: a float's square is exact there and no sum overflows, so the total is finite exactly where every gradient
// is, and its rounding to float does not depend on the order of the sum (but for one in 10^8).  The last CTA adds the CTAs' sums
// in the order of their numbers.
template <int GRAD>
__global__ void __launch_bounds__(kAdamThreads, kNormCtasPerSm) grad_norm_kernel(char* ws, Layout lay, float max_norm, const float* loss_scale, float* norm_out) {
    ptx::grid_handover();
    Control* control = reinterpret_cast<Control*>(ws);
    double* partials = reinterpret_cast<double*>(ws + lay.partials);
    __shared__ Tensor table[kTable];
    __shared__ double shared[kAdamThreads / 32];
    __shared__ bool last;
    const int lane = threadIdx.x & 31;
    double sums[4] = {};
    auto add = [&](const uint4& u, int dtype) {
        float2 f[2];
        widen4(u, dtype, f);
        sums[0] = fma((double)f[0].x, (double)f[0].x, sums[0]);
        sums[1] = fma((double)f[0].y, (double)f[0].y, sums[1]);
        sums[2] = fma((double)f[1].x, (double)f[1].x, sums[2]);
        sums[3] = fma((double)f[1].y, (double)f[1].y, sums[3]);
    };
    for_chunks(ws, lay, table, [&](int64_t first, int count) {
        for (int i0 = 0; i0 < count; i0 += kNormUnroll) {
            uint4 u[kNormUnroll][2];
#pragma unroll
            for (int i = 0; i < kNormUnroll; ++i) {
                u[i][0] = u[i][1] = make_uint4(0u, 0u, 0u, 0u);
                if (i0 + i >= count) continue;
                const Tensor& x = table[i0 + i];
                const Block block(x, first + (int64_t)(i0 + i) * gridDim.x);
                const int size = (GRAD == kMixed ? x.grad_dtype : GRAD) == EQL_FP32 ? 4 : 2;
                const char* g = (const char*)x.grad + (block.base + lane * 4) * size;
                if (block.count == kBlock) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) u[i][h] = size == 4 ? load_raw4<4>(g + h * kRun * 4) : load_raw4<2>(g + h * kRun * 2);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int mine = block.count - h * kRun - lane * 4;
                        u[i][h] = size == 4 ? load_some4<4>(g + h * kRun * 4, mine) : load_some4<2>(g + h * kRun * 2, mine);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kNormUnroll; ++i) {
                const int dtype = GRAD != kMixed ? GRAD : table[i0 + i < count ? i0 + i : i0].grad_dtype;
                add(u[i][0], dtype);
                add(u[i][1], dtype);
            }
        }
    });
    double sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    sum = cta_sum(sum, shared);
    if (threadIdx.x == 0) {
        partials[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(&control->norm_ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kAdamThreads) sum += __ldcg(partials + i);
    sum = cta_sum(sum, shared);
    if (threadIdx.x == 0) {
        const float scale = loss_scale ? *loss_scale : 1.0f;
        const float norm = (float)(sqrt(sum) / (double)scale);
        const float factor = __fdiv_rn(fminf(1.0f, __fdiv_rn(max_norm, __fadd_rn(norm, 1e-6f))), scale);
        const bool fine = isfinite(norm) && isfinite(scale) && scale > 0.0f && isfinite(factor);
        control->norm = norm;
        control->skip = fine ? 0 : 1;
        control->factor = fine ? factor : 0.0f;
        control->norm_ticket = 0;
        if (norm_out) *norm_out = norm;
    }
}

__global__ void set_step_kernel(char* ws, int64_t step) {
    Control* control = reinterpret_cast<Control*>(ws);
    control->step = step;
    control->factor = 1.0f;
    control->skip = 0;
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline bool known_dtype(int d) { return d == EQL_FP32 || d == EQL_FP16 || d == EQL_BF16; }
inline int64_t chunks_of(int64_t numel) { return (numel + kChunk - 1) / kChunk; }

eql_status_t layout(const eql_adamw_tensor_t* tensors, int count, int state_bits, Layout* lay) {
    if (!tensors || count < 1 || (state_bits != 8 && state_bits != 32)) return EQL_ERR_INVALID_ARG;
    if (count > 1 << 20) return EQL_ERR_UNSUPPORTED;
    int64_t chunks = 0;
    for (int i = 0; i < count; ++i) {
        if (tensors[i].numel < 0) return EQL_ERR_INVALID_ARG;
        if (tensors[i].numel > (int64_t)1 << 40) return EQL_ERR_UNSUPPORTED;
        chunks += chunks_of(tensors[i].numel);
    }
    if (chunks > ((int64_t)1 << 31) - 1) return EQL_ERR_UNSUPPORTED;
    lay->n_chunks = chunks;
    lay->partials = kWsAlign;
    lay->tensors = lay->partials + kMaxNormCtas * sizeof(double);
    lay->chunks = align_up(lay->tensors + (size_t)count * sizeof(Tensor), kWsAlign);
    lay->total = align_up(lay->chunks + (size_t)chunks * sizeof(int32_t), kWsAlign);
    return EQL_OK;
}

struct Range {
    uintptr_t begin, end;
    bool written;
};

eql_status_t check_tensor(const eql_adamw_tensor_t& t, int state_bits, Range* ranges, int* n) {
    if (!known_dtype(t.param_dtype) || !known_dtype(t.grad_dtype)) return EQL_ERR_INVALID_ARG;
    if (!(t.weight_decay >= 0.0f) || !std::isfinite(t.weight_decay) || !std::isfinite(t.lr_scale)) return EQL_ERR_INVALID_ARG;
    if (t.numel == 0) return EQL_OK;
    if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq) return EQL_ERR_INVALID_ARG;
    if ((state_bits == 8) != (t.exp_avg_scale != nullptr) || (state_bits == 8) != (t.exp_avg_sq_scale != nullptr)) return EQL_ERR_INVALID_ARG;
    if (!aligned(t.param, 16) || !aligned(t.master, 16) || !aligned(t.grad, 16) || !aligned(t.exp_avg, 16) || !aligned(t.exp_avg_sq, 16) ||
        !aligned(t.exp_avg_scale, 4) || !aligned(t.exp_avg_sq_scale, 4))
        return EQL_ERR_ALIGNMENT;
    const int64_t blocks = (t.numel + kBlock - 1) / kBlock;
    auto add = [&](const void* p, int64_t bytes, bool written) {
        if (p) ranges[(*n)++] = Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written};
    };
    add(t.param, t.numel * (t.param_dtype == EQL_FP32 ? 4 : 2), true);
    add(t.master, t.numel * 4, true);
    add(t.grad, t.numel * (t.grad_dtype == EQL_FP32 ? 4 : 2), false);
    add(t.exp_avg, t.numel * (state_bits / 8), true);
    add(t.exp_avg_sq, t.numel * (state_bits / 8), true);
    add(t.exp_avg_scale, blocks * 4, true);
    add(t.exp_avg_sq_scale, blocks * 4, true);
    return EQL_OK;
}

// Whether a pointer is memory of `device` (or none): a kernel that met another one would fault.
bool on_device(const void* p, int device) {
    if (!p) return true;
    cudaPointerAttributes a{};
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) { cudaGetLastError(); return false; }
    return a.type == cudaMemoryTypeManaged || (a.type == cudaMemoryTypeDevice && a.device == device);
}
bool on_device(const eql_adamw_tensor_t& t, int device) {
    for (const void* p : {(const void*)t.param, (const void*)t.master, (const void*)t.grad, (const void*)t.exp_avg, (const void*)t.exp_avg_sq,
                          (const void*)t.exp_avg_scale, (const void*)t.exp_avg_sq_scale})
        if (!on_device(p, device)) return false;
    return true;
}
// Whether a kernel on `device` can reach a scalar (or there is none): pinned memory of the host counts, pageable memory does not.
bool reachable(const void* p, int device) {
    if (!p) return true;
    cudaPointerAttributes a{};
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) { cudaGetLastError(); return false; }
    return a.type == cudaMemoryTypeManaged || a.type == cudaMemoryTypeHost || (a.type == cudaMemoryTypeDevice && a.device == device);
}
// Calls that wait for a stream cannot be captured.
eql_status_t not_capturing(cudaStream_t s) {
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(s, &capturing) != cudaSuccess) return EQL_ERR_CUDA;
    return capturing == cudaStreamCaptureStatusNone ? EQL_OK : EQL_ERR_INVALID_ARG;
}

// Whether a written range shares bytes with any other.
bool ranges_clash(Range* ranges, int n) {
    std::sort(ranges, ranges + n, [](const Range& a, const Range& b) { return a.begin < b.begin; });
    uintptr_t end = 0, end_written = 0;
    for (int i = 0; i < n; ++i) {
        if (ranges[i].begin < (ranges[i].written ? end : end_written)) return true;
        end = std::max(end, ranges[i].end);
        if (ranges[i].written) end_written = std::max(end_written, ranges[i].end);
    }
    return false;
}

}  // namespace
}  // namespace eql

// The host object behind eqlinear_adamw_t.
struct eqlinear_adamw_s {
    int device, num_sms, state_bits;
    int grad_dtype, param_dtype;      // all tensors', or kMixed
    char* ws;
    eql::Layout lay;
};

namespace {

using namespace eql;

using StepKernel = void (*)(char*, Layout, Rates);
template <int BITS, int GRAD>
StepKernel step_kernel(int param_dtype) {
    return param_dtype == EQL_FP32 ? adamw_kernel<BITS, GRAD, EQL_FP32> : param_dtype == EQL_FP16 ? adamw_kernel<BITS, GRAD, EQL_FP16> : adamw_kernel<BITS, GRAD, EQL_BF16>;
}
template <int BITS>
StepKernel step_kernel(int grad_dtype, int param_dtype) {
    if (grad_dtype == kMixed || param_dtype == kMixed) return adamw_kernel<BITS, kMixed, kMixed>;
    return grad_dtype == EQL_FP32 ? step_kernel<BITS, EQL_FP32>(param_dtype) : grad_dtype == EQL_FP16 ? step_kernel<BITS, EQL_FP16>(param_dtype)
                                                                                                    : step_kernel<BITS, EQL_BF16>(param_dtype);
}

eql_status_t check_optimiser(eqlinear_adamw_t opt) {
    if (!opt) return EQL_ERR_INVALID_ARG;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return EQL_ERR_CUDA;
    return dev == opt->device ? EQL_OK : EQL_ERR_INVALID_ARG;
}

}  // namespace

extern "C" {

eql_status_t eqlinear_adamw_workspace_bytes(const eql_adamw_tensor_t* tensors, int count, int state_bits, size_t* bytes) {
    if (!bytes) return EQL_ERR_INVALID_ARG;
    Layout lay{};
    if (eql_status_t st = layout(tensors, count, state_bits, &lay); st != EQL_OK) return st;
    *bytes = lay.total;
    return EQL_OK;
}

eql_status_t eqlinear_adamw(eqlinear_adamw_t* opt, const eql_adamw_tensor_t* tensors, int count, int state_bits, void* workspace,
                            size_t workspace_bytes, void* stream) {
    if (!opt) return EQL_ERR_INVALID_ARG;
    *opt = nullptr;
    Layout lay{};
    if (eql_status_t st = layout(tensors, count, state_bits, &lay); st != EQL_OK) return st;
    if (!workspace) return EQL_ERR_INVALID_ARG;
    if (!aligned(workspace, kWsAlign)) return EQL_ERR_ALIGNMENT;
    if (workspace_bytes < lay.total) return EQL_ERR_WORKSPACE;
    Range* ranges = new (std::nothrow) Range[(size_t)count * 7 + 1];
    if (!ranges) return EQL_ERR_INVALID_ARG;
    int n = 0;
    ranges[n++] = Range{(uintptr_t)workspace, (uintptr_t)workspace + lay.total, true};
    eql_status_t st = EQL_OK;
    for (int i = 0; i < count && st == EQL_OK; ++i) st = check_tensor(tensors[i], state_bits, ranges, &n);
    if (st == EQL_OK && ranges_clash(ranges, n)) st = EQL_ERR_INVALID_ARG;
    delete[] ranges;
    if (st != EQL_OK) return st;

    int dev = 0, major = 0, sms = kNumSMs;
    if (cudaGetDevice(&dev) != cudaSuccess) return EQL_ERR_CUDA;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) return EQL_ERR_CUDA;
    if (major != 10) return EQL_ERR_ARCH;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return EQL_ERR_CUDA;
    if (!on_device(workspace, dev)) return EQL_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i)
        if (tensors[i].numel > 0 && !on_device(tensors[i], dev)) return EQL_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    if (eql_status_t c = not_capturing(s); c != EQL_OK) return c;

    char* image = static_cast<char*>(std::calloc(1, lay.total));
    if (!image) return EQL_ERR_INVALID_ARG;
    reinterpret_cast<Control*>(image)->factor = 1.0f;
    Tensor* table = reinterpret_cast<Tensor*>(image + lay.tensors);
    int32_t* chunk_tensor = reinterpret_cast<int32_t*>(image + lay.chunks);
    int64_t chunk = 0;
    for (int i = 0; i < count; ++i) {
        const eql_adamw_tensor_t& t = tensors[i];
        table[i] = Tensor{t.param, (float*)t.master, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale, t.numel, (int32_t)chunk,
                          t.param_dtype, t.grad_dtype, t.weight_decay, t.lr_scale, 0};
        for (int64_t k = chunks_of(t.numel); k > 0; --k) chunk_tensor[chunk++] = i;
    }
    cudaError_t e = cudaMemcpyAsync(workspace, image, lay.total, cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    std::free(image);
    if (e != cudaSuccess) return EQL_ERR_CUDA;
    eqlinear_adamw_s* o = new (std::nothrow) eqlinear_adamw_s{dev, sms, state_bits, tensors[0].grad_dtype, tensors[0].param_dtype, (char*)workspace, lay};
    if (!o) return EQL_ERR_INVALID_ARG;
    for (int i = 1; i < count; ++i) {
        if (tensors[i].grad_dtype != o->grad_dtype) o->grad_dtype = kMixed;
        if (tensors[i].param_dtype != o->param_dtype) o->param_dtype = kMixed;
    }
    *opt = o;
    return EQL_OK;
}

eql_status_t eqlinear_adamw_clip(eqlinear_adamw_t opt, float max_norm, const float* loss_scale, float* norm, void* stream) {
    if (eql_status_t st = check_optimiser(opt); st != EQL_OK) return st;
    if (!(max_norm > 0.0f)) return EQL_ERR_INVALID_ARG;
    if (!aligned(loss_scale, 4) || !aligned(norm, 4)) return EQL_ERR_ALIGNMENT;
    if (!reachable(loss_scale, opt->device) || !reachable(norm, opt->device)) return EQL_ERR_INVALID_ARG;
    const int64_t most = std::min(opt->num_sms * kNormCtasPerSm, kMaxNormCtas);
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min(opt->lay.n_chunks, most));
    const auto kernel = opt->grad_dtype == kMixed ? grad_norm_kernel<kMixed> : opt->grad_dtype == EQL_FP32 ? grad_norm_kernel<EQL_FP32>
                        : opt->grad_dtype == EQL_FP16 ? grad_norm_kernel<EQL_FP16> : grad_norm_kernel<EQL_BF16>;
    cudaError_t e = launch_overlapped(kernel, dim3(grid), dim3(kAdamThreads), 0, (cudaStream_t)stream, opt->ws, opt->lay, max_norm,
                                      loss_scale, norm);
    return e == cudaSuccess ? EQL_OK : EQL_ERR_CUDA;
}

eql_status_t eqlinear_adamw_step(eqlinear_adamw_t opt, double lr, double beta1, double beta2, double eps, const float* lr_device, void* stream) {
    if (eql_status_t st = check_optimiser(opt); st != EQL_OK) return st;
    if (!(lr >= 0.0) || !std::isfinite((float)lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return EQL_ERR_INVALID_ARG;
    if (!((float)eps >= FLT_MIN) || !std::isfinite((float)eps)) return EQL_ERR_INVALID_ARG;
    if (!aligned(lr_device, 4)) return EQL_ERR_ALIGNMENT;
    if (!reachable(lr_device, opt->device)) return EQL_ERR_INVALID_ARG;
    const Rates r{(float)lr, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, 1.0f, std::log(beta1), std::log(beta2), lr_device};
    const int64_t most = (int64_t)opt->num_sms * step_ctas_per_sm(opt->state_bits);
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min(opt->lay.n_chunks, most));
    const auto kernel = opt->state_bits == 8 ? step_kernel<8>(opt->grad_dtype, opt->param_dtype) : step_kernel<32>(opt->grad_dtype, opt->param_dtype);
    cudaError_t e = launch_overlapped(kernel, dim3(grid), dim3(kAdamThreads), 0, (cudaStream_t)stream, opt->ws, opt->lay, r);
    return e == cudaSuccess ? EQL_OK : EQL_ERR_CUDA;
}

eql_status_t eqlinear_adamw_set_step(eqlinear_adamw_t opt, int64_t step, void* stream) {
    if (eql_status_t st = check_optimiser(opt); st != EQL_OK) return st;
    if (step < 0) return EQL_ERR_INVALID_ARG;
    set_step_kernel<<<1, 1, 0, (cudaStream_t)stream>>>(opt->ws, step);
    return cudaGetLastError() == cudaSuccess ? EQL_OK : EQL_ERR_CUDA;
}

eql_status_t eqlinear_adamw_info(eqlinear_adamw_t opt, eql_adamw_info_t* info, void* stream) {
    if (eql_status_t st = check_optimiser(opt); st != EQL_OK) return st;
    if (!info) return EQL_ERR_INVALID_ARG;
    if (eql_status_t st = not_capturing((cudaStream_t)stream); st != EQL_OK) return st;
    Control c{};
    if (cudaMemcpyAsync(&c, opt->ws, sizeof(c), cudaMemcpyDeviceToHost, (cudaStream_t)stream) != cudaSuccess) return EQL_ERR_CUDA;
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return EQL_ERR_CUDA;
    *info = eql_adamw_info_t{c.step, c.skipped, c.norm, c.skip};
    return EQL_OK;
}

eql_status_t eqlinear_adamw_destroy(eqlinear_adamw_t opt) {
    delete opt;
    return EQL_OK;
}

}  // extern "C"
