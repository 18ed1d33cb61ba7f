// Group norm of small units: an instance's part of one group fits the registers of a warp or a part of one (the norm of every token by
// itself above all).
//
// A unit of up to 128 vectors of 16 bytes belongs to 1, 2, 4, ... 32 lanes, whichever holds a vector each; larger ones give a lane up to
// four.  x is read once: mean, then the squared distances from it, then the result, all from registers.  A warp stays with its
// groups and walks over the instances, the next one's vectors on their way while one is computed; what belongs to a column (gamma,
// beta, in the backward pass the sums for dgamma and dbeta) stays in registers for the whole walk: one value a vector where its
// elements are of one channel, else gamma and beta as packed as x.
#include "groupnorm_common.cuh"

namespace eql {
namespace {

// Threads of a CTA and CTAs that are resident together, by the registers that NV vectors a lane need.
constexpr int threads_for(int nv) { return nv <= 2 ? 256 : 128; }
constexpr int forward_ctas(int nv, bool tuple) { return nv == 1 ? 4 : nv == 2 ? (tuple ? 4 : 3) : nv == 3 ? (tuple ? 6 : 4) : tuple ? 5 : 3; }
constexpr int gradient_ctas(int nv, int sums) { return nv == 1 ? 3 : nv == 2 ? 2 : sums > 1 ? 2 : nv == 3 ? 4 : 3; }

// Gamma (or beta) of the columns of one vector: TUPLE, where they are of one channel, as one float, else in x's own type.
template <typename IO, bool TUPLE>
struct Parameter {
    uint4 packed;
    float one;
    __device__ __forceinline__ void get(const IO* p, float none, int element, int T) {
        if (TUPLE) {
            one = p ? NormIo<IO>::one(p, element / T) : none;
        } else {
            float2 f[NormIo<IO>::kVec / 2];
#pragma unroll
            for (int j = 0; j < NormIo<IO>::kVec; ++j) (&f[j / 2].x)[j % 2] = p ? NormIo<IO>::one(p, (element + j) / T) : none;
            packed = NormIo<IO>::narrow(f);
        }
    }
    __device__ __forceinline__ void widen(float2* f) const {
        if (TUPLE) {
#pragma unroll
            for (int j = 0; j < NormIo<IO>::kVec / 2; ++j) f[j] = pair(one);
        } else {
            NormIo<IO>::widen(packed, f);
        }
    }
};

__device__ __forceinline__ float lanes_sum(float v, int lanes) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
        if (d < lanes) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// Where a thread stands: its lane in the unit, its group, its first instance.
struct Seat {
    int lane, group, chair;   // chair: which of the CTA's units at a time
    int64_t b, step;
    bool active;
};
__device__ __forceinline__ Seat seat(const NormShape& s, const WarpNorm& w) {
    Seat t;
    t.lane = threadIdx.x % w.lanes;
    t.chair = threadIdx.x / w.lanes;
    const int block = blockIdx.x % (unsigned)w.group_blocks, cta = blockIdx.x / (unsigned)w.group_blocks;
    t.group = block * w.groups + t.chair % w.groups;
    t.active = t.chair < w.groups * w.instances && t.group < s.groups;
    t.b = (int64_t)cta * w.instances + t.chair / w.groups;
    t.step = (int64_t)(gridDim.x / (unsigned)w.group_blocks) * w.instances;
    return t;
}

template <typename IO, int NV>
struct Vectors {
    int at[NV];               // offset of a vector from its instance's first
    int row[NV];
    __device__ __forceinline__ Vectors(const NormShape& s, const WarpNorm& w, const Seat& t) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = t.lane + w.lanes * k;
            row[k] = t.active && i < w.unit ? i / w.vectors : INT_MAX;
            at[k] = (int)(i / w.vectors) * s.vectors + t.group * w.vectors + i % w.vectors;
        }
    }
    __device__ __forceinline__ void load(uint4* raw, const uint4* x, const NormShape& s, int64_t b, int n) const {
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (row[k] < n) raw[k] = x[b * s.S * s.vectors + at[k]];
    }
};

template <typename IO, int ACT, int NV, bool TUPLE>
__global__ void __launch_bounds__(threads_for(NV), forward_ctas(NV, TUPLE)) warp_norm_kernel(NormShape s, WarpNorm w, const uint4* x, const IO* gammas,
                                                                                      const IO* betas, const int32_t* lengths, uint4* y, float2* stats) {
    constexpr int V = NormIo<IO>::kVec, P = V / 2;
    ptx::grid_handover();
    const Seat t = seat(s, w);
    const Vectors<IO, NV> v(s, w, t);
    Parameter<IO, TUPLE> gamma[NV], beta[NV];
    uint4 next[NV];
    const int64_t rounds = (s.B + t.step - 1) / t.step;      // the same for all: lanes of one warp may hold units of different instances
    int64_t b = t.b;
    int n = b < s.B ? (int)positions_of(lengths, b, s.S) : 0;
    v.load(next, x, s, b, n);
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (v.row[k] != INT_MAX) {
            const int e = (t.group * w.vectors + (t.lane + w.lanes * k) % w.vectors) * V;
            gamma[k].get(gammas, 1.0f, e, s.T);
            beta[k].get(betas, 0.0f, e, s.T);
        }
    for (int64_t i = 0; i < rounds; ++i, b += t.step) {
        const int now = n;
        float2 f[NV][P], sum = pair(0.0f), squares = pair(0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                NormIo<IO>::widen(next[k], f[k]);
#pragma unroll
                for (int j = 0; j < P; ++j) sum = add2(sum, f[k][j]);
            }
        n = b + t.step < s.B ? (int)positions_of(lengths, b + t.step, s.S) : 0;
        v.load(next, x, s, b + t.step, n);
        const float count = (float)now * s.width;
        const float share = count > 0.0f ? reciprocal(count) : 0.0f;
        const float mean = lanes_sum(sum.x + sum.y, w.lanes) * share;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    f[k][j] = sub2(f[k][j], pair(mean));
                    squares = fma2(f[k][j], f[k][j], squares);
                }
            }
        const float rstd = rsqrtf(fmaf(lanes_sum(squares.x + squares.y, w.lanes), share, s.eps));
        if (stats && t.active && t.lane == 0 && b < s.B) stats[b * s.groups + t.group] = make_float2(mean, rstd);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                float2 ga[P], be[P];
                gamma[k].widen(ga);
                beta[k].widen(be);
#pragma unroll
                for (int j = 0; j < P; ++j) f[k][j] = activate<ACT, TUPLE>(fma2(f[k][j], mul2(ga[j], pair(rstd)), be[j]));
                y[b * s.S * s.vectors + v.at[k]] = NormIo<IO>::narrow(f[k]);
            }
    }
}

// SUMS: pairs of partial sums that a vector keeps for dgamma and dbeta: 1 where its elements are of one channel, half of its pairs where
// they are of two, else all.
template <typename IO, int ACT, int NV, int SUMS>
__global__ void __launch_bounds__(threads_for(NV), gradient_ctas(NV, SUMS)) warp_gradient_kernel(NormShape s, WarpNorm w, const uint4* x, const uint4* dy,
                                                                                          const IO* gammas, const IO* betas, const int32_t* lengths,
                                                                                          const float2* stats, uint4* dx, float2* parts) {
    constexpr int V = NormIo<IO>::kVec, P = V / 2;
    extern __shared__ float2 shared[];
    ptx::grid_handover();
    const Seat t = seat(s, w);
    const Vectors<IO, NV> v(s, w, t);
    Parameter<IO, SUMS == 1> gamma[NV], beta[NV];
    uint4 nx[NV], nd[NV];
    float2 db[NV][SUMS] = {}, dg[NV][SUMS] = {};
    const int64_t rounds = (s.B + t.step - 1) / t.step;
    int64_t b = t.b;
    int n = b < s.B ? (int)positions_of(lengths, b, s.S) : 0;
    float2 st = t.active && b < s.B ? stats[b * s.groups + t.group] : make_float2(0.0f, 0.0f);
    v.load(nx, x, s, b, n);
    v.load(nd, dy, s, b, n);
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (v.row[k] != INT_MAX) {
            const int e = (t.group * w.vectors + (t.lane + w.lanes * k) % w.vectors) * V;
            gamma[k].get(gammas, 1.0f, e, s.T);
            beta[k].get(betas, 0.0f, e, s.T);
        }
    for (int64_t i = 0; i < rounds; ++i, b += t.step) {
        const int now = n;
        const float mean = st.x, rstd = st.y;
        float2 xc[NV][P], dz[NV][P], t1 = pair(0.0f), t2 = pair(0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                NormIo<IO>::widen(nx[k], xc[k]);
                NormIo<IO>::widen(nd[k], dz[k]);
            }
        const bool more = b + t.step < s.B;
        n = more ? (int)positions_of(lengths, b + t.step, s.S) : 0;
        if (t.active && more) st = stats[(b + t.step) * s.groups + t.group];
        v.load(nx, x, s, b + t.step, n);
        v.load(nd, dy, s, b + t.step, n);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                float2 ga[P], be[P];
                gamma[k].widen(ga);
                if (ACT != EQL_ACT_NONE) beta[k].widen(be);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float2 xh = mul2(sub2(xc[k][j], pair(mean)), pair(rstd));
                    if (ACT != EQL_ACT_NONE) dz[k][j] = mul2(dz[k][j], slope<ACT, (SUMS < P)>(fma2(xh, ga[j], be[j])));
                    float2 &b_sum = db[k][j * SUMS / P], &g_sum = dg[k][j * SUMS / P];
                    b_sum = add2(b_sum, dz[k][j]);
                    g_sum = fma2(dz[k][j], xh, g_sum);
                    dz[k][j] = mul2(dz[k][j], ga[j]);         // from here on times gamma
                    t1 = add2(t1, dz[k][j]);
                    t2 = fma2(dz[k][j], xh, t2);
                    xc[k][j] = xh;
                }
            }
        const float count = (float)now * s.width;
        const float share = count > 0.0f ? reciprocal(count) : 0.0f;
        // dx = rstd * gamma * dz - rstd * s1 - xh * rstd * s2
        const float2 off1 = pair(-rstd * share * lanes_sum(t1.x + t1.y, w.lanes)), off2 = pair(-rstd * share * lanes_sum(t2.x + t2.y, w.lanes));
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
#pragma unroll
                for (int j = 0; j < P; ++j) dz[k][j] = fma2(xc[k][j], off2, fma2(dz[k][j], pair(rstd), off1));
                dx[b * s.S * s.vectors + v.at[k]] = NormIo<IO>::narrow(dz[k]);
            }
    }
    // The CTA's share of dbeta and dgamma: every thread's partial sums side by side in shared memory, then a thread a channel.
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (t.chair < w.groups * w.instances && t.lane + w.lanes * k < w.unit) {
            float2* to = shared + (t.chair * w.unit + t.lane + w.lanes * k) * w.sums;
#pragma unroll
            for (int j = 0; j < SUMS; ++j) {
                if (w.sums > SUMS) {                          // (each half of a pair is a channel's)
                    to[2 * j] = make_float2(db[k][j].x, dg[k][j].x);
                    to[2 * j + 1] = make_float2(db[k][j].y, dg[k][j].y);
                } else {
                    to[j] = make_float2(db[k][j].x + db[k][j].y, dg[k][j].x + dg[k][j].y);
                }
            }
        }
    __syncthreads();
    const int each = s.C / s.groups, runs = s.T * w.sums / V, row = w.vectors * w.sums;
    const int block = blockIdx.x % (unsigned)w.group_blocks, cta = blockIdx.x / (unsigned)w.group_blocks;
    const int groups = min(w.groups, s.groups - block * w.groups);
    for (int c = threadIdx.x; c < groups * each; c += blockDim.x) {
        float2 sum = make_float2(0.0f, 0.0f);
        for (int instance = 0; instance < w.instances; ++instance) {
            const float2* from = shared + (instance * w.groups + c / each) * w.unit * w.sums + c % each * runs;
            for (int r = 0; r < (int)s.S; ++r)
                for (int e = 0; e < runs; ++e) {
                    const float2 p = from[r * row + e];
                    sum.x += p.x; sum.y += p.y;
                }
        }
        parts[(int64_t)cta * s.C + block * w.groups * each + c] = sum;
    }
}

}  // namespace

// Units whose rows are whole vectors, no more than 128 in all: with eight vectors a lane the kernels need 250 registers, and too few
// warps are left to keep the memory busy.
WarpNorm warp_norm_plan(const NormShape& s, eql_dtype_t dtype, bool backward) {
    WarpNorm w{};
    const int V = dtype == EQL_FP32 ? 4 : 8;
    if (s.width % V != 0 || s.S * (s.width / V) > 128) return w;
    w.vectors = s.width / V;
    w.unit = (int)s.S * w.vectors;
    w.lanes = 1;
    while (w.lanes < 32 && w.lanes < w.unit) w.lanes *= 2;
    w.each = (w.unit + w.lanes - 1) / w.lanes;
    const int chairs = threads_for(w.each) / w.lanes;
    w.groups = s.groups < chairs ? s.groups : chairs;
    w.instances = chairs / w.groups;
    w.group_blocks = (s.groups + w.groups - 1) / w.groups;
    w.sums = V / run_length(s.T, V);
    w.shared_bytes = backward ? w.groups * w.instances * w.unit * w.sums * 8 : 0;
    // CTAs that are resident together walk over the instances, all about the same number
    const int together = kNumSMs * (backward ? gradient_ctas(w.each, w.sums) : forward_ctas(w.each, w.sums == 1));
    const int64_t wanted = (s.B + w.instances - 1) / w.instances, most = together > w.group_blocks ? together / w.group_blocks : 1;
    const int64_t rounds = (wanted + most - 1) / most;
    w.ctas = (int)((wanted + rounds - 1) / rounds);
    w.supported = true;
    return w;
}

template <typename F>
static cudaError_t dispatch_vectors(int each, F&& f) {
    switch (each) {
        case 1: return f(std::integral_constant<int, 1>{});
        case 2: return f(std::integral_constant<int, 2>{});
        case 3: return f(std::integral_constant<int, 3>{});
        default: return f(std::integral_constant<int, 4>{});
    }
}

cudaError_t launch_warp_norm(const NormShape& s, const WarpNorm& w, eql_dtype_t dtype, const void* x, const void* gamma, const void* beta,
                             const int32_t* lengths, void* y, float* stats, cudaStream_t stream) {
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            return dispatch_vectors(w.each, [&](auto nv) {
                constexpr int NV = decltype(nv)::value;
                return launch_overlapped(w.sums == 1 ? warp_norm_kernel<IO, ACT, NV, true> : warp_norm_kernel<IO, ACT, NV, false>,
                                         dim3((unsigned)(w.ctas * w.group_blocks)), dim3(threads_for(NV)), 0, stream, s, w, (const uint4*)x, (const IO*)gamma,
                                         (const IO*)beta, lengths, (uint4*)y, (float2*)stats);
            });
        });
    });
}

cudaError_t launch_warp_gradient(const NormShape& s, const WarpNorm& w, eql_dtype_t dtype, const void* x, const void* dy, const void* gamma,
                                 const void* beta, const int32_t* lengths, const float* stats, void* dx, float* parts, cudaStream_t stream) {
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        constexpr int P = NormIo<IO>::kVec / 2;
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            return dispatch_vectors(w.each, [&](auto nv) {
                constexpr int NV = decltype(nv)::value;
                auto launch = [&](auto kernel, SmemLimitOnce& limit) -> cudaError_t {
                    if (cudaError_t e = limit.ensure(kernel, kWarpNormShared); e != cudaSuccess) return e;
                    return launch_overlapped(kernel, dim3((unsigned)(w.ctas * w.group_blocks)), dim3(threads_for(NV)), w.shared_bytes, stream, s, w,
                                             (const uint4*)x, (const uint4*)dy, (const IO*)gamma, (const IO*)beta, lengths, (const float2*)stats,
                                             (uint4*)dx, (float2*)parts);
                };
                static SmemLimitOnce limits[3];
                if (w.sums == 1) return launch(warp_gradient_kernel<IO, ACT, NV, 1>, limits[0]);
                if (w.sums == 2 && P > 2) return launch(warp_gradient_kernel<IO, ACT, NV, 2>, limits[1]);
                return launch(warp_gradient_kernel<IO, ACT, NV, P>, limits[2]);
            });
        });
    });
}

}  // namespace eql
