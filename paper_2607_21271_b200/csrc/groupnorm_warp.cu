// Group norm of small units: an instance's part of one group fits the registers of a warp or a part of one (the norm of every token by
// itself above all).
//
// A unit of up to 128 vectors of 16 bytes belongs to 1, 2, 4, ... 32 lanes, whichever holds a vector each; larger ones give a lane up to
// four.  x is read once: mean, then the squared distances from it, then the result, all from registers.  A warp stays with its
// groups and walks over the instances, the next one's vectors on their way while one is computed; what belongs to a column (gamma,
// beta, in the backward pass the sums for dgamma and dbeta) stays in registers for the whole walk, gamma and beta as packed as x.
#include "groupnorm_common.cuh"

namespace eql {
namespace {

constexpr int kThreads = 256;

// V elements of gamma (or beta) of the columns of one vector, in x's own type.
template <typename IO>
__device__ __forceinline__ uint4 pack_parameter(const IO* p, float none, int element, int T) {
    float2 f[NormIo<IO>::kVec / 2];
#pragma unroll
    for (int j = 0; j < NormIo<IO>::kVec; ++j) (&f[j / 2].x)[j % 2] = p ? NormIo<IO>::one(p, (element + j) / T) : none;
    return NormIo<IO>::narrow(f);
}

__device__ __forceinline__ float lanes_sum(float v, int lanes) {
    for (int d = lanes >> 1; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
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

template <typename IO, int ACT, int NV>
__global__ void __launch_bounds__(kThreads) warp_norm_kernel(NormShape s, WarpNorm w, const uint4* x, const IO* gammas, const IO* betas,
                                                             const int32_t* lengths, uint4* y, float2* stats) {
    constexpr int V = NormIo<IO>::kVec;
    ptx::grid_handover();
    const Seat t = seat(s, w);
    const Vectors<IO, NV> v(s, w, t);
    uint4 gamma[NV], beta[NV], raw[NV], next[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (v.row[k] != INT_MAX) {
            const int e = (t.group * w.vectors + (t.lane + w.lanes * k) % w.vectors) * V;
            gamma[k] = pack_parameter(gammas, 1.0f, e, s.T);
            beta[k] = pack_parameter(betas, 0.0f, e, s.T);
        }
    const int64_t rounds = (s.B + t.step - 1) / t.step;      // the same for all: lanes of one warp may hold units of different instances
    int64_t b = t.b;
    int n = b < s.B ? (int)positions_of(lengths, b, s.S) : 0;
    v.load(next, x, s, b, n);
    for (int64_t i = 0; i < rounds; ++i, b += t.step) {
        const int now = n;
#pragma unroll
        for (int k = 0; k < NV; ++k) raw[k] = next[k];
        n = b + t.step < s.B ? (int)positions_of(lengths, b + t.step, s.S) : 0;
        v.load(next, x, s, b + t.step, n);
        float2 sum = pair(0.0f), squares = pair(0.0f);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                float2 f[V / 2];
                NormIo<IO>::widen(raw[k], f);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) sum = add2(sum, f[j]);
            }
        const float count = (float)now * s.width;
        const float share = count > 0.0f ? __fdividef(1.0f, count) : 0.0f;
        const float mean = lanes_sum(sum.x + sum.y, w.lanes) * share;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                float2 f[V / 2];
                NormIo<IO>::widen(raw[k], f);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    const float2 d = sub2(f[j], pair(mean));
                    squares = fma2(d, d, squares);
                }
            }
        const float rstd = 1.0f / sqrtf(lanes_sum(squares.x + squares.y, w.lanes) * share + s.eps);
        if (stats && t.active && t.lane == 0 && b < s.B) stats[b * s.groups + t.group] = make_float2(mean, rstd);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                float2 f[V / 2], ga[V / 2], be[V / 2];
                NormIo<IO>::widen(raw[k], f);
                NormIo<IO>::widen(gamma[k], ga);
                NormIo<IO>::widen(beta[k], be);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) f[j] = activate<ACT>(fma2(mul2(sub2(f[j], pair(mean)), pair(rstd)), ga[j], be[j]));
                y[b * s.S * s.vectors + v.at[k]] = NormIo<IO>::narrow(f);
            }
    }
}

// SUMS: pairs of partial sums a vector keeps for dgamma and dbeta, 1 where its elements are of one channel, else all.
template <typename IO, int ACT, int NV, int SUMS>
__global__ void __launch_bounds__(kThreads) warp_gradient_kernel(NormShape s, WarpNorm w, const uint4* x, const uint4* dy, const IO* gammas,
                                                                 const IO* betas, const int32_t* lengths, const float2* stats, uint4* dx, float2* parts) {
    constexpr int V = NormIo<IO>::kVec;
    extern __shared__ float2 shared[];
    ptx::grid_handover();
    const Seat t = seat(s, w);
    const Vectors<IO, NV> v(s, w, t);
    uint4 gamma[NV], beta[NV], rx[NV], rd[NV], nx[NV], nd[NV];
    float2 db[NV][SUMS] = {}, dg[NV][SUMS] = {};
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (v.row[k] != INT_MAX) {
            const int e = (t.group * w.vectors + (t.lane + w.lanes * k) % w.vectors) * V;
            gamma[k] = pack_parameter(gammas, 1.0f, e, s.T);
            beta[k] = pack_parameter(betas, 0.0f, e, s.T);
        }
    const int64_t rounds = (s.B + t.step - 1) / t.step;
    int64_t b = t.b;
    int n = b < s.B ? (int)positions_of(lengths, b, s.S) : 0;
    float2 st = t.active && b < s.B ? stats[b * s.groups + t.group] : make_float2(0.0f, 0.0f);
    v.load(nx, x, s, b, n);
    v.load(nd, dy, s, b, n);
    for (int64_t i = 0; i < rounds; ++i, b += t.step) {
        const int now = n;
        const float mean = st.x, rstd = st.y;
#pragma unroll
        for (int k = 0; k < NV; ++k) { rx[k] = nx[k]; rd[k] = nd[k]; }
        const bool more = b + t.step < s.B;
        n = more ? (int)positions_of(lengths, b + t.step, s.S) : 0;
        if (t.active && more) st = stats[(b + t.step) * s.groups + t.group];
        v.load(nx, x, s, b + t.step, n);
        v.load(nd, dy, s, b + t.step, n);
        float2 t1 = pair(0.0f), t2 = pair(0.0f), xh[V / 2], dz[V / 2];
        auto both = [&](int k, const float2* ga) {             // xh and dz of a vector, dz not yet times gamma
            float2 be[V / 2];
            NormIo<IO>::widen(rx[k], xh);
            NormIo<IO>::widen(rd[k], dz);
            if (ACT != EQL_ACT_NONE) NormIo<IO>::widen(beta[k], be);
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                xh[j] = mul2(sub2(xh[j], pair(mean)), pair(rstd));
                if (ACT != EQL_ACT_NONE) dz[j] = mul2(dz[j], slope<ACT>(fma2(xh[j], ga[j], be[j])));
            }
        };
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                float2 ga[V / 2];
                NormIo<IO>::widen(gamma[k], ga);
                both(k, ga);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    db[k][j % SUMS] = add2(db[k][j % SUMS], dz[j]);
                    dg[k][j % SUMS] = fma2(dz[j], xh[j], dg[k][j % SUMS]);
                    const float2 scaled = mul2(dz[j], ga[j]);
                    t1 = add2(t1, scaled);
                    t2 = fma2(scaled, xh[j], t2);
                }
            }
        const float count = (float)now * s.width;
        const float share = count > 0.0f ? __fdividef(1.0f, count) : 0.0f;
        const float s1 = lanes_sum(t1.x + t1.y, w.lanes) * share, s2 = lanes_sum(t2.x + t2.y, w.lanes) * share;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (v.row[k] < now) {
                float2 ga[V / 2], f[V / 2];
                NormIo<IO>::widen(gamma[k], ga);
                both(k, ga);
#pragma unroll
                for (int j = 0; j < V / 2; ++j)
                    f[j] = mul2(pair(rstd), fma2(xh[j], pair(-s2), fma2(ga[j], dz[j], pair(-s1))));
                dx[b * s.S * s.vectors + v.at[k]] = NormIo<IO>::narrow(f);
            }
    }
    // The CTA's share of dbeta and dgamma: every thread's partial sums side by side in shared memory, then a thread a channel.
#pragma unroll
    for (int k = 0; k < NV; ++k)
        if (t.chair < w.groups * w.instances && t.lane + w.lanes * k < w.unit) {
            float2* to = shared + (t.chair * w.unit + t.lane + w.lanes * k) * w.sums;
#pragma unroll
            for (int j = 0; j < SUMS; ++j) {
                if (SUMS == 1) {
                    to[0] = make_float2(db[k][0].x + db[k][0].y, dg[k][0].x + dg[k][0].y);
                } else {
                    to[2 * j] = make_float2(db[k][j].x, dg[k][j].x);
                    to[2 * j + 1] = make_float2(db[k][j].y, dg[k][j].y);
                }
            }
        }
    __syncthreads();
    const int each = s.C / s.groups, runs = SUMS == 1 ? s.T / V : s.T, row = w.vectors * w.sums;
    const int block = blockIdx.x % (unsigned)w.group_blocks, cta = blockIdx.x / (unsigned)w.group_blocks;
    const int groups = min(w.groups, s.groups - block * w.groups);
    for (int c = threadIdx.x; c < groups * each; c += kThreads) {
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
    if (w.each == 3) w.each = 4;
    const int chairs = kThreads / w.lanes;
    w.groups = s.groups < chairs ? s.groups : chairs;
    w.instances = chairs / w.groups;
    w.group_blocks = (s.groups + w.groups - 1) / w.groups;
    w.sums = s.T % V == 0 ? 1 : V;
    w.shared_bytes = backward ? w.groups * w.instances * w.unit * w.sums * 8 : 0;
    // CTAs that are resident together walk over the instances
    const int64_t wanted = (s.B + w.instances - 1) / w.instances, most = ((int64_t)kNumSMs * (backward ? 2 : 4) + w.group_blocks - 1) / w.group_blocks;
    w.ctas = (int)(wanted < most ? wanted : most);
    w.supported = true;
    return w;
}

cudaError_t launch_warp_norm(const NormShape& s, const WarpNorm& w, eql_dtype_t dtype, const void* x, const void* gamma, const void* beta,
                             const int32_t* lengths, void* y, float* stats, cudaStream_t stream) {
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            auto kernel = w.each == 1 ? warp_norm_kernel<IO, ACT, 1> : w.each == 2 ? warp_norm_kernel<IO, ACT, 2> :
                          warp_norm_kernel<IO, ACT, 4>;
            return launch_overlapped(kernel, dim3((unsigned)(w.ctas * w.group_blocks)), dim3(kThreads), 0, stream, s, w, (const uint4*)x,
                                     (const IO*)gamma, (const IO*)beta, lengths, (uint4*)y, (float2*)stats);
        });
    });
}

cudaError_t launch_warp_gradient(const NormShape& s, const WarpNorm& w, eql_dtype_t dtype, const void* x, const void* dy, const void* gamma,
                                 const void* beta, const int32_t* lengths, const float* stats, void* dx, float* parts, cudaStream_t stream) {
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        constexpr int V = NormIo<IO>::kVec;
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            auto launch = [&](auto kernel, SmemLimitOnce& limit) -> cudaError_t {
                if (cudaError_t e = limit.ensure(kernel, kWarpNormShared); e != cudaSuccess) return e;
                return launch_overlapped(kernel, dim3((unsigned)(w.ctas * w.group_blocks)), dim3(kThreads), w.shared_bytes, stream, s, w,
                                         (const uint4*)x, (const uint4*)dy, (const IO*)gamma, (const IO*)beta, lengths, (const float2*)stats,
                                         (uint4*)dx, (float2*)parts);
            };
            static SmemLimitOnce limits[6];
            if (w.sums == 1)
                return w.each == 1 ? launch(warp_gradient_kernel<IO, ACT, 1, 1>, limits[0]) : w.each == 2 ? launch(warp_gradient_kernel<IO, ACT, 2, 1>, limits[1])
                                   : launch(warp_gradient_kernel<IO, ACT, 4, 1>, limits[2]);
            return w.each == 1 ? launch(warp_gradient_kernel<IO, ACT, 1, V / 2>, limits[3]) : w.each == 2 ? launch(warp_gradient_kernel<IO, ACT, 2, V / 2>, limits[4])
                               : launch(warp_gradient_kernel<IO, ACT, 4, V / 2>, limits[5]);
        });
    });
}

}  // namespace eql
