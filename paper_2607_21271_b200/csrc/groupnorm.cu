// Group norm with an activation, forward and backward: kernels that go through global memory between statistics and result, and the
// C entry points.
//
// These kernels take every shape.  A CTA works on a piece of up to 256 vectors of a row, over a range of rows of one instance; a thread
// stays with one vector column, so that what belongs to a column (statistics, gamma, sums) lies in its registers however
// the borders of channels and groups fall.  Forward: moments of every range of rows, piece and group, their merging, and a pass that
// applies them; backward: sums of dz and dz * xh of every range, piece and channel, their sums, and a pass that applies them.
// x (and dy) are read twice; the second pass begins with the rows that the first one read last, some of which L2 still holds.
#include <cmath>

#include "groupnorm_common.cuh"

namespace eql {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;    // vectors a thread has on their way
// CTAs resident together, by the registers that the kernels then may use.
constexpr int range_ctas(int n, int P) { return n < P ? 4 : 2; }

// Row ranges and pieces of an instance.
struct Ranges {
    int pieces, ranges;       // pieces of a row, ranges of rows
    int64_t rows;             // rows of a range
    int parts;                // groups (forward) or channels (backward) that a piece touches at most
    float* partials;          // float2 [B][ranges][pieces][parts]
    float* groups;            // float2 [B][groups]: forward mean and rstd, backward the two means that dx takes off
    float* channels;          // float2 [B][C], backward
};

struct Place {
    int64_t b, row0;
    int rows, range, piece, vector, count, lane, lanes;      // count: vectors of the piece
    bool active;
    __device__ __forceinline__ int rows_of(int l) const { return l < rows ? (rows - l + lanes - 1) / lanes : 0; }
};
// blockIdx.x = (b * ranges + range) * pieces + piece
__device__ __forceinline__ Place place(const NormShape& s, const Ranges& g, const int32_t* lengths, unsigned index) {
    Place p;
    const int64_t unit = index / (unsigned)g.pieces;
    p.piece = (int)(index % (unsigned)g.pieces);
    const int first = p.piece * kThreads;
    p.count = min(kThreads, s.vectors - first);
    p.b = unit / g.ranges;
    p.range = (int)(unit % g.ranges);
    p.lanes = kThreads / p.count;
    p.lane = threadIdx.x / p.count;
    p.vector = first + threadIdx.x % p.count;
    p.active = p.lane < p.lanes;
    p.row0 = p.range * g.rows;
    const int64_t left = positions_of(lengths, p.b, s.S) - p.row0;
    p.rows = (int)(left < 0 ? 0 : left < g.rows ? left : g.rows);
    return p;
}

// Part `k` (group or channel) of `each` elements, within a piece whose elements are [first, first + count): its own elements.
struct Part {
    int begin, end;
    __device__ __forceinline__ Part(int k, int each, int first, int count) : begin(max(k * each, first) - first), end(min((k + 1) * each, first + count) - first) {}
};

// A column of vectors `step` apart, kUnroll of them in flight; use(i) for each.
template <int N, typename Load, typename Use>
__device__ __forceinline__ void walk(int count, Load&& load, Use&& use) {
    int i = 0;
    for (; i + kUnroll <= count; i += kUnroll) {
        uint4 u[kUnroll][N];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) load(i + k, u[k]);
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) use(i + k, u[k]);
    }
    for (; i < count; ++i) {
        uint4 u[N];
        load(i, u);
        use(i, u);
    }
}

template <typename IO>
__global__ void __launch_bounds__(kThreads, 4) part_moments_kernel(NormShape s, Ranges g, const uint4* x, const int32_t* lengths) {
    constexpr int V = NormIo<IO>::kVec;
    ptx::grid_handover();
    __shared__ float2 shared[kThreads * V];
    const Place p = place(s, g, lengths, blockIdx.x);
    RunningMoments<V / 2> m;
    if (p.active) {
        const uint4* at = x + (p.b * s.S + p.row0 + p.lane) * s.vectors + p.vector;
        const int64_t step = (int64_t)p.lanes * s.vectors;
        walk<1>(p.rows_of(p.lane), [&](int i, uint4* u) { u[0] = at[i * step]; },
                [&](int, const uint4* u) {
                    float2 f[V / 2];
                    NormIo<IO>::widen(u[0], f);
                    m.add(f);
                });
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            shared[threadIdx.x * V + 2 * j] = make_float2(m.mean[j].x, m.m2[j].x);
            shared[threadIdx.x * V + 2 * j + 1] = make_float2(m.mean[j].y, m.m2[j].y);
        }
    }
    __syncthreads();
    // a column over the lanes of rows, then (its values in lane 0's place) a warp a group
    const int first = p.piece * kThreads * V, count = p.count * V;
    for (int c = threadIdx.x; c < count; c += kThreads) {
        Moments all{0.0f, 0.0f, 0.0f};
        for (int l = 0; l < p.lanes && l < p.rows; ++l) {
            const float2 v = shared[l * count + c];
            all = merge(all, Moments{(float)p.rows_of(l), v.x, v.y});
        }
        shared[c] = make_float2(all.mean, all.m2);
    }
    __syncthreads();
    const int group0 = first / s.width, groups = (first + count - 1) / s.width - group0 + 1;
    float2* out = reinterpret_cast<float2*>(g.partials) + ((p.b * g.ranges + p.range) * g.pieces + p.piece) * g.parts;
    for (int k = threadIdx.x >> 5; k < groups; k += kThreads / 32) {
        const Part part(group0 + k, s.width, first, count);
        Moments all{0.0f, 0.0f, 0.0f};
        for (int c = part.begin + (threadIdx.x & 31); c < part.end; c += 32) all = merge(all, Moments{(float)p.rows, shared[c].x, shared[c].y});
        all = warp_merge(all);
        if ((threadIdx.x & 31) == 0) out[k] = make_float2(all.mean, all.m2);
    }
}

// One CTA an instance and group.
__global__ void __launch_bounds__(kThreads) group_moments_kernel(NormShape s, Ranges g, int V, const int32_t* lengths, float* stats) {
    ptx::grid_handover();
    __shared__ Moments shared[kThreads / 32];
    const int64_t b = blockIdx.x / (unsigned)s.groups;
    const int group = (int)(blockIdx.x % (unsigned)s.groups), size = kThreads * V;
    const int64_t n = positions_of(lengths, b, s.S);
    const int piece0 = group * s.width / size, pieces = ((group + 1) * s.width - 1) / size - piece0 + 1;
    Moments all{0.0f, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < g.ranges * pieces; i += kThreads) {
        const int range = i / pieces, piece = piece0 + i % pieces;
        const int64_t left = n - range * g.rows;
        const Part part(group, s.width, piece * size, min(size, s.D - piece * size));
        const float rows = (float)(left < 0 ? 0 : left < g.rows ? left : g.rows);
        const float2 v = reinterpret_cast<const float2*>(g.partials)[((b * g.ranges + range) * g.pieces + piece) * g.parts + group - piece * size / s.width];
        all = merge(all, Moments{rows * (part.end - part.begin), v.x, v.y});
    }
    all = warp_merge(all);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) all = merge(all, shared[w]);
        const float2 out = make_float2(all.mean, rstd_of(all, s.eps));
        reinterpret_cast<float2*>(g.groups)[blockIdx.x] = out;
        if (stats) reinterpret_cast<float2*>(stats)[blockIdx.x] = out;
    }
}

// What a thread keeps of its column, N: see Runs.
template <typename IO, int N>
struct Column {
    static constexpr int V = NormIo<IO>::kVec, P = V / 2;
    using R = Runs<N, P>;
    R mean, rstd, scale, beta;                                // scale: rstd * gamma
    __device__ __forceinline__ Column(const NormShape& s, const float2* stats, const IO* gammas, const IO* betas, int64_t b, int vector) {
        const int channel = vector * V / s.T, group = vector * V / s.width;
        R::each(channel, vector * V - channel * s.T, s.T, [&](int e, int c) {
            scale.set(e, gammas ? NormIo<IO>::one(gammas, c) : 1.0f);
            beta.set(e, betas ? NormIo<IO>::one(betas, c) : 0.0f);
        });
        R::each(group, vector * V - group * s.width, s.width, [&](int e, int g) {
            const float2 st = stats[b * s.groups + g];
            mean.set(e, st.x);
            rstd.set(e, st.y);
        });
#pragma unroll
        for (int j = 0; j < N; ++j) scale.v[j] = mul2(scale.v[j], rstd.v[j]);
    }
    // x - mean and dz of a vector
    template <int ACT>
    __device__ __forceinline__ void gradient(const uint4* u, float2* xc, float2* dz) const {
        NormIo<IO>::widen(u[0], xc);
        NormIo<IO>::widen(u[1], dz);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            xc[j] = sub2(xc[j], mean.of(j));
            if (ACT != EQL_ACT_NONE) dz[j] = mul2(dz[j], slope<ACT, (N < P)>(fma2(xc[j], scale.of(j), beta.of(j))));
        }
    }
};

template <typename IO, int ACT, int N>
__global__ void __launch_bounds__(kThreads, range_ctas(N, NormIo<IO>::kVec / 2)) apply_kernel(NormShape s, Ranges g, const uint4* x, const IO* gamma, const IO* beta,
                                                         const int32_t* lengths, uint4* y) {
    constexpr int V = NormIo<IO>::kVec;
    ptx::grid_handover();
    const Place p = place(s, g, lengths, gridDim.x - 1 - blockIdx.x);
    if (!p.active || p.lane >= p.rows) return;
    const Column<IO, N> c(s, reinterpret_cast<const float2*>(g.groups), gamma, beta, p.b, p.vector);
    const int64_t at = (p.b * s.S + p.row0 + p.lane) * s.vectors + p.vector, step = (int64_t)p.lanes * s.vectors;
    walk<1>(p.rows_of(p.lane), [&](int i, uint4* u) { u[0] = x[at + i * step]; },
            [&](int i, const uint4* u) {
                float2 f[V / 2];
                NormIo<IO>::widen(u[0], f);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) f[j] = activate<ACT, (N < V / 2)>(fma2(sub2(f[j], c.mean.of(j)), c.scale.of(j), c.beta.of(j)));
                y[at + i * step] = NormIo<IO>::narrow(f);
            });
}

template <typename IO, int ACT, int N>
__global__ void __launch_bounds__(kThreads, range_ctas(N, NormIo<IO>::kVec / 2)) part_sums_kernel(NormShape s, Ranges g, const uint4* x, const uint4* dy, const IO* gamma, const IO* beta,
                                                             const int32_t* lengths, const float* stats) {
    constexpr int V = NormIo<IO>::kVec;
    ptx::grid_handover();
    __shared__ float2 shared[kThreads * V];
    const Place p = place(s, g, lengths, blockIdx.x);
    float2 db[V / 2] = {}, dg[V / 2] = {};
    if (p.active && p.lane < p.rows) {
        const Column<IO, N> c(s, reinterpret_cast<const float2*>(stats), gamma, beta, p.b, p.vector);
        const int64_t at = (p.b * s.S + p.row0 + p.lane) * s.vectors + p.vector, step = (int64_t)p.lanes * s.vectors;
        walk<2>(p.rows_of(p.lane), [&](int i, uint4* u) { u[0] = x[at + i * step]; u[1] = dy[at + i * step]; },
                [&](int, const uint4* u) {
                    float2 xc[V / 2], dz[V / 2];
                    c.template gradient<ACT>(u, xc, dz);
#pragma unroll
                    for (int j = 0; j < V / 2; ++j) {
                        db[j] = add2(db[j], dz[j]);
                        dg[j] = fma2(dz[j], xc[j], dg[j]);
                    }
                });
#pragma unroll
        for (int j = 0; j < V / 2; ++j) dg[j] = mul2(dg[j], c.rstd.of(j));
    }
    if (p.active) {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
            shared[threadIdx.x * V + 2 * j] = make_float2(db[j].x, dg[j].x);
            shared[threadIdx.x * V + 2 * j + 1] = make_float2(db[j].y, dg[j].y);
        }
    }
    __syncthreads();
    const int first = p.piece * kThreads * V, count = p.count * V;
    const int channel0 = first / s.T, channels = (first + count - 1) / s.T - channel0 + 1;
    float2* out = reinterpret_cast<float2*>(g.partials) + ((p.b * g.ranges + p.range) * g.pieces + p.piece) * g.parts;
    for (int k = threadIdx.x; k < channels; k += kThreads) {
        const Part part(channel0 + k, s.T, first, count);
        float2 all = make_float2(0.0f, 0.0f);
        for (int l = 0; l < p.lanes && l < p.rows; ++l)
            for (int c = part.begin; c < part.end; ++c) all = add2(all, shared[l * count + c]);
        out[k] = all;
    }
}

// A channel of an instance over all ranges (and the two pieces that a channel can lie in): eight channels a CTA and 32 chains.
__global__ void __launch_bounds__(kThreads) channel_sums_kernel(NormShape s, Ranges g, int V) {
    ptx::grid_handover();
    __shared__ float2 shared[kThreads];
    const int blocks = (s.C + 7) / 8, size = kThreads * V;
    const int64_t b = blockIdx.x / (unsigned)blocks;
    const int channel = (int)(blockIdx.x % (unsigned)blocks) * 8 + (threadIdx.x & 7);
    float2 sum = make_float2(0.0f, 0.0f);
    if (channel < s.C) {
        const int piece0 = channel * s.T / size, pieces = ((channel + 1) * s.T - 1) / size - piece0 + 1;
        for (int piece = piece0; piece < piece0 + pieces; ++piece) {
            const float2* from = reinterpret_cast<const float2*>(g.partials) + (b * g.ranges * g.pieces + piece) * g.parts + channel - piece * size / s.T;
            const int64_t step = (int64_t)g.pieces * g.parts;
#pragma unroll 8
            for (int range = threadIdx.x >> 3; range < g.ranges; range += kThreads / 8) sum = add2(sum, from[range * step]);
        }
    }
    shared[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 8 && channel < s.C) {
        for (int k = 1; k < kThreads / 8; ++k) sum = add2(sum, shared[k * 8 + threadIdx.x]);
        reinterpret_cast<float2*>(g.channels)[b * s.C + channel] = sum;
    }
}

__device__ __forceinline__ float2 warp_sum(float2 v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
    }
    return v;
}

// One warp an instance and group.
template <typename IO>
__global__ void __launch_bounds__(kThreads) group_sums_kernel(NormShape s, Ranges g, const IO* gamma, const int32_t* lengths) {
    ptx::grid_handover();
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (unit >= s.B * s.groups) return;
    const int64_t b = unit / s.groups;
    const int group = (int)(unit % s.groups), each = s.C / s.groups;
    float2 total = make_float2(0.0f, 0.0f);
    for (int k = threadIdx.x & 31; k < each; k += 32) {
        const int channel = group * each + k;
        const float w = gamma ? NormIo<IO>::one(gamma, channel) : 1.0f;
        total = fma2(pair(w), reinterpret_cast<const float2*>(g.channels)[b * s.C + channel], total);
    }
    total = warp_sum(total);
    if ((threadIdx.x & 31) == 0) {
        const float n = (float)positions_of(lengths, b, s.S) * s.width;
        reinterpret_cast<float2*>(g.groups)[unit] = n > 0.0f ? make_float2(total.x / n, total.y / n) : make_float2(0.0f, 0.0f);
    }
}

template <typename IO, int ACT, int N>
__global__ void __launch_bounds__(kThreads, range_ctas(N, NormIo<IO>::kVec / 2)) apply_gradient_kernel(NormShape s, Ranges g, const uint4* x, const uint4* dy, const IO* gamma, const IO* beta,
                                                                  const int32_t* lengths, const float* stats, uint4* dx) {
    constexpr int V = NormIo<IO>::kVec;
    ptx::grid_handover();
    const Place p = place(s, g, lengths, gridDim.x - 1 - blockIdx.x);
    if (!p.active || p.lane >= p.rows) return;
    const Column<IO, N> c(s, reinterpret_cast<const float2*>(stats), gamma, beta, p.b, p.vector);
    // dx = dz * (rstd * gamma) - (x - mean) * (rstd * rstd * second) - rstd * first
    Runs<N, V / 2> off1, off2;
    const int group = p.vector * V / s.width;
    Runs<N, V / 2>::each(group, p.vector * V - group * s.width, s.width, [&](int e, int k) {
        const float2 v = reinterpret_cast<const float2*>(g.groups)[p.b * s.groups + k];
        off1.set(e, -v.x);
        off2.set(e, -v.y);
    });
#pragma unroll
    for (int j = 0; j < N; ++j) {
        off1.v[j] = mul2(off1.v[j], c.rstd.v[j]);
        off2.v[j] = mul2(mul2(off2.v[j], c.rstd.v[j]), c.rstd.v[j]);
    }
    const int64_t at = (p.b * s.S + p.row0 + p.lane) * s.vectors + p.vector, step = (int64_t)p.lanes * s.vectors;
    walk<2>(p.rows_of(p.lane), [&](int i, uint4* u) { u[0] = x[at + i * step]; u[1] = dy[at + i * step]; },
            [&](int i, const uint4* u) {
                float2 xc[V / 2], dz[V / 2];
                c.template gradient<ACT>(u, xc, dz);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) xc[j] = fma2(xc[j], off2.of(j), fma2(dz[j], c.scale.of(j), off1.of(j)));
                dx[at + i * step] = NormIo<IO>::narrow(xc);
            });
}

// dgamma and dbeta: the sum over `parts` rows of float2 [parts][C], eight channels a CTA and 32 chains.
__global__ void __launch_bounds__(kThreads) parameter_sums_kernel(const float2* parts, int64_t count, int C, float* dgamma, float* dbeta) {
    ptx::grid_handover();
    __shared__ float2 shared[kThreads];
    const int channel = blockIdx.x * 8 + (threadIdx.x & 7);
    float2 sum = make_float2(0.0f, 0.0f);
    if (channel < C) {
#pragma unroll 8
        for (int64_t i = threadIdx.x >> 3; i < count; i += kThreads / 8) sum = add2(sum, parts[i * C + channel]);
    }
    shared[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 8 && channel < C) {
        for (int k = 1; k < kThreads / 8; ++k) { sum.x += shared[k * 8 + threadIdx.x].x; sum.y += shared[k * 8 + threadIdx.x].y; }
        if (dbeta) dbeta[channel] = sum.x;
        if (dgamma) dgamma[channel] = sum.y;
    }
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t elem(int dtype) { return dtype == EQL_FP32 ? 4 : 2; }

eql_status_t check_norm(const eql_groupnorm_t* n, NormShape* s) {
    if (!n) return EQL_ERR_INVALID_ARG;
    if (n->dtype != EQL_FP32 && n->dtype != EQL_FP16 && n->dtype != EQL_BF16) return EQL_ERR_INVALID_ARG;
    if (n->T < 1 || n->C < 1 || n->groups < 1 || n->C % n->groups != 0) return EQL_ERR_INVALID_ARG;
    if (n->act < EQL_ACT_NONE || n->act > EQL_ACT_SILU || !(n->eps > 0.0f) || !std::isfinite(n->eps)) return EQL_ERR_INVALID_ARG;
    if (n->batch < 0 || n->positions < 0) return EQL_ERR_INVALID_ARG;
    const int64_t most = ((int64_t)1 << 31) - 1024, D = (int64_t)n->C * n->T;
    if (n->T > 64 || D > (1 << 20) || n->batch > most || n->positions > most || n->batch * n->positions > most) return EQL_ERR_UNSUPPORTED;
    if (D * elem(n->dtype) % 16 != 0) return EQL_ERR_ALIGNMENT;
    *s = NormShape{n->T, n->C, n->groups, n->act, (int)D, (int)(D / n->groups), (int)(D * elem(n->dtype) / 16), n->batch, n->positions, n->eps};
    return EQL_OK;
}

// Ranges of rows so that a launch fills the device once, of 32 rows at least.  (One map of 65536 x 1024 half precision, forward and
// backward: one filling 228 us, two 240.)
Ranges range_plan(const NormShape& s, eql_dtype_t dtype, bool backward, char* scratch, size_t* bytes) {
    Ranges g{};
    const int V = dtype == EQL_FP32 ? 4 : 8;
    g.pieces = (s.vectors + kThreads - 1) / kThreads;
    const int64_t wanted = 4 * kNumSMs / (s.B * g.pieces) > 0 ? 4 * kNumSMs / (s.B * g.pieces) : 1;
    const int64_t most = s.S / 32 > 1 ? s.S / 32 : 1;
    const int64_t ranges = wanted < most ? wanted : most;
    g.rows = (s.S + ranges - 1) / ranges;
    g.ranges = (int)((s.S + g.rows - 1) / g.rows);
    const int elements = s.D < kThreads * V ? s.D : kThreads * V, each = backward ? s.T : s.width;
    g.parts = (elements + each - 2) / each + 1;
    size_t off = 0;
    g.partials = (float*)(scratch + off);  off += align_up((size_t)s.B * g.ranges * g.pieces * g.parts * 8, kWsAlign);
    g.groups = (float*)(scratch + off);    off += align_up((size_t)s.B * s.groups * 8, kWsAlign);
    g.channels = (float*)(scratch + off);  if (backward) off += align_up((size_t)s.B * s.C * 8, kWsAlign);
    *bytes = off;
    return g;
}

// How one direction of a norm runs, by its shape alone.
struct NormPlan {
    WarpNorm warp;
    ResidentNorm resident;
    Ranges ranges;            // where no other kernel takes the shape
    size_t scratch_bytes;
    bool fits;                // its launches
};
NormPlan norm_plan(const NormShape& s, eql_dtype_t dtype, bool backward, char* scratch) {
    NormPlan p{};
    p.fits = true;
    p.warp = warp_norm_plan(s, dtype, backward);
    if (p.warp.supported) {
        p.scratch_bytes = backward ? align_up((size_t)p.warp.ctas * s.C * 8, kWsAlign) : 0;
        return p;
    }
    p.resident = resident_norm_plan(s, dtype, backward);
    if (p.resident.supported) {
        p.scratch_bytes = backward ? align_up((size_t)p.resident.instances * p.resident.cluster * s.C * 8, kWsAlign) : 0;
        return p;
    }
    p.ranges = range_plan(s, dtype, backward, scratch, &p.scratch_bytes);
    p.fits = s.B * p.ranges.ranges * p.ranges.pieces <= INT32_MAX && s.B * s.groups <= INT32_MAX && s.B * ((s.C + 7) / 8) <= INT32_MAX;
    return p;
}

cudaError_t launch_parameter_sums(const float* parts, int64_t count, int C, float* dgamma, float* dbeta, cudaStream_t stream) {
    if (!dgamma && !dbeta) return cudaSuccess;
    return launch_overlapped(parameter_sums_kernel, dim3((unsigned)((C + 7) / 8)), dim3(kThreads), 0, stream, (const float2*)parts, count, C, dgamma, dbeta);
}

cudaError_t run_ranges(const NormShape& s, const Ranges& g, eql_dtype_t dtype, const void* x, const void* gamma, const void* beta, const int32_t* lengths,
                       void* y, float* stats, cudaStream_t st) {
    const int64_t grid = s.B * g.ranges * g.pieces, units = s.B * s.groups;
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        cudaError_t err = launch_overlapped(part_moments_kernel<IO>, dim3((unsigned)grid), dim3(kThreads), 0, st, s, g, (const uint4*)x, lengths);
        if (err == cudaSuccess) err = launch_overlapped(group_moments_kernel, dim3((unsigned)units), dim3(kThreads), 0, st, s, g, NormIo<IO>::kVec, lengths, stats);
        if (err != cudaSuccess) return err;
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value, V = NormIo<IO>::kVec;
            return launch_overlapped(runs_of(s.T, V) == 1 ? apply_kernel<IO, ACT, 1> : runs_of(s.T, V) == 2 ? apply_kernel<IO, ACT, 2> : apply_kernel<IO, ACT, V / 2>, dim3((unsigned)grid), dim3(kThreads), 0, st, s, g, (const uint4*)x,
                                     (const IO*)gamma, (const IO*)beta, lengths, (uint4*)y);
        });
    });
}

cudaError_t run_ranges_gradient(const NormShape& s, const Ranges& g, eql_dtype_t dtype, const void* x, const void* dy, const void* gamma, const void* beta,
                                const int32_t* lengths, const float* stats, void* dx, float* dgamma, float* dbeta, cudaStream_t st) {
    const int64_t grid = s.B * g.ranges * g.pieces, units = s.B * s.groups;
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value, V = NormIo<IO>::kVec;
            const int runs = runs_of(s.T, V);
            cudaError_t err = launch_overlapped(runs == 1 ? part_sums_kernel<IO, ACT, 1> : runs == 2 ? part_sums_kernel<IO, ACT, 2> : part_sums_kernel<IO, ACT, V / 2>, dim3((unsigned)grid), dim3(kThreads), 0, st, s, g, (const uint4*)x,
                                                (const uint4*)dy, (const IO*)gamma, (const IO*)beta, lengths, stats);
            if (err == cudaSuccess)
                err = launch_overlapped(channel_sums_kernel, dim3((unsigned)(s.B * ((s.C + 7) / 8))), dim3(kThreads), 0, st, s, g, NormIo<IO>::kVec);
            if (err == cudaSuccess)
                err = launch_overlapped(group_sums_kernel<IO>, dim3((unsigned)((units + kThreads / 32 - 1) / (kThreads / 32))), dim3(kThreads), 0, st, s, g,
                                        (const IO*)gamma, lengths);
            if (err == cudaSuccess)
                err = launch_overlapped(runs == 1 ? apply_gradient_kernel<IO, ACT, 1> : runs == 2 ? apply_gradient_kernel<IO, ACT, 2> : apply_gradient_kernel<IO, ACT, V / 2>, dim3((unsigned)grid), dim3(kThreads), 0, st, s, g, (const uint4*)x,
                                        (const uint4*)dy, (const IO*)gamma, (const IO*)beta, lengths, stats, (uint4*)dx);
            return err == cudaSuccess ? launch_parameter_sums(g.channels, s.B, s.C, dgamma, dbeta, st) : err;
        });
    });
}

// Whether [a, a + na) and [b, b + nb) share bytes.
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t p = (uintptr_t)a, q = (uintptr_t)b;
    return p < q + nb && q < p + na;
}

eql_status_t check_scratch(const void* scratch, size_t bytes, size_t need) {
    if (need == 0) return EQL_OK;
    if (!scratch) return EQL_ERR_INVALID_ARG;
    if (!aligned(scratch, kWsAlign)) return EQL_ERR_ALIGNMENT;
    return bytes < need ? EQL_ERR_WORKSPACE : EQL_OK;
}

}  // namespace
}  // namespace eql

using namespace eql;

extern "C" {

eql_status_t eqlinear_groupnorm_scratch_bytes(const eql_groupnorm_t* norm, size_t* bytes) {
    if (!bytes) return EQL_ERR_INVALID_ARG;
    NormShape s;
    if (eql_status_t st = check_norm(norm, &s); st != EQL_OK) return st;
    *bytes = 0;
    if (s.B > 0 && s.S > 0) {
        const eql_dtype_t dtype = (eql_dtype_t)norm->dtype;
        const size_t fwd = norm_plan(s, dtype, false, nullptr).scratch_bytes, bwd = norm_plan(s, dtype, true, nullptr).scratch_bytes;
        *bytes = fwd > bwd ? fwd : bwd;
    }
    return EQL_OK;
}

eql_status_t eqlinear_groupnorm_fwd(const eql_groupnorm_t* norm, const void* x, const void* gamma, const void* beta, const int32_t* lengths,
                                    void* y, float* stats, void* scratch, size_t scratch_bytes, void* stream) {
    NormShape s;
    if (eql_status_t st = check_norm(norm, &s); st != EQL_OK) return st;
    if (s.B == 0 || s.S == 0) return EQL_OK;
    if (!x || !y) return EQL_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(gamma, 16) || !aligned(beta, 16) || !aligned(lengths, 16) || !aligned(stats, 16))
        return EQL_ERR_ALIGNMENT;
    const size_t size = (size_t)s.B * s.S * s.vectors * 16;
    if (overlap(x, size, y, size)) return EQL_ERR_INVALID_ARG;
    const eql_dtype_t dtype = (eql_dtype_t)norm->dtype;
    const NormPlan p = norm_plan(s, dtype, false, (char*)scratch);
    if (!p.fits) return EQL_ERR_UNSUPPORTED;
    if (eql_status_t st = check_scratch(scratch, scratch_bytes, p.scratch_bytes); st != EQL_OK) return st;
    const cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = p.warp.supported ? launch_warp_norm(s, p.warp, dtype, x, gamma, beta, lengths, y, stats, st)
                          : p.resident.supported ? launch_resident_norm(s, p.resident, dtype, x, gamma, beta, lengths, y, stats, st)
                                                 : run_ranges(s, p.ranges, dtype, x, gamma, beta, lengths, y, stats, st);
    return e == cudaSuccess ? EQL_OK : EQL_ERR_CUDA;
}

eql_status_t eqlinear_groupnorm_bwd(const eql_groupnorm_t* norm, const void* x, const void* dy, const void* gamma, const void* beta,
                                    const int32_t* lengths, const float* stats, void* dx, void* dgamma, void* dbeta,
                                    void* scratch, size_t scratch_bytes, void* stream) {
    NormShape s;
    if (eql_status_t st = check_norm(norm, &s); st != EQL_OK) return st;
    if (!aligned(dgamma, 16) || !aligned(dbeta, 16)) return EQL_ERR_ALIGNMENT;
    if (dgamma && dbeta && overlap(dgamma, s.C * sizeof(float), dbeta, s.C * sizeof(float))) return EQL_ERR_INVALID_ARG;
    const cudaStream_t st = (cudaStream_t)stream;
    if (s.B == 0 || s.S == 0) {
        if (dgamma && cudaMemsetAsync(dgamma, 0, s.C * sizeof(float), st) != cudaSuccess) return EQL_ERR_CUDA;
        if (dbeta && cudaMemsetAsync(dbeta, 0, s.C * sizeof(float), st) != cudaSuccess) return EQL_ERR_CUDA;
        return EQL_OK;
    }
    if (!x || !dy || !stats || !dx) return EQL_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(dy, 16) || !aligned(dx, 16) || !aligned(gamma, 16) || !aligned(beta, 16) || !aligned(lengths, 16) ||
        !aligned(stats, 16))
        return EQL_ERR_ALIGNMENT;
    const size_t size = (size_t)s.B * s.S * s.vectors * 16;
    if (overlap(x, size, dx, size) || overlap(dy, size, dx, size)) return EQL_ERR_INVALID_ARG;
    const eql_dtype_t dtype = (eql_dtype_t)norm->dtype;
    const NormPlan p = norm_plan(s, dtype, true, (char*)scratch);
    if (!p.fits) return EQL_ERR_UNSUPPORTED;
    if (eql_status_t e = check_scratch(scratch, scratch_bytes, p.scratch_bytes); e != EQL_OK) return e;
    cudaError_t e;
    if (p.warp.supported) {
        e = launch_warp_gradient(s, p.warp, dtype, x, dy, gamma, beta, lengths, stats, dx, (float*)scratch, st);
        if (e == cudaSuccess) e = launch_parameter_sums((const float*)scratch, p.warp.ctas, s.C, (float*)dgamma, (float*)dbeta, st);
    } else if (p.resident.supported) {
        e = launch_resident_gradient(s, p.resident, dtype, x, dy, gamma, beta, lengths, stats, dx, (float*)scratch, st);
        if (e == cudaSuccess)
            e = launch_parameter_sums((const float*)scratch, (int64_t)p.resident.instances * p.resident.cluster, s.C, (float*)dgamma, (float*)dbeta, st);
    } else {
        e = run_ranges_gradient(s, p.ranges, dtype, x, dy, gamma, beta, lengths, stats, dx, (float*)dgamma, (float*)dbeta, st);
    }
    return e == cudaSuccess ? EQL_OK : EQL_ERR_CUDA;
}

}  // extern "C"
