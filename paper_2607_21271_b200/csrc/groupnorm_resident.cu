// Group norm with an instance's groups resident in shared memory: x (and dy) are read once.
//
// A unit is a block of whole groups of one instance, at least 128 bytes of every row where there are as many.  It belongs to one CTA, or to a
// cluster whose CTAs hold a range of its rows each; what they have to tell each other is one triple (forward) or pair (backward) a
// group, written into every CTA's shared memory.  A thread stays with one 16-byte column, which it copies asynchronously into slots of its own: no
// barrier stands between copy and use, and as many bytes are in flight as shared memory holds.
// What bounds it is the memory; several CTAs to an SM overlap one's reading with another's writing.
#include "groupnorm_common.cuh"

namespace eql {
namespace {

constexpr int kMaxCluster = 8;

__device__ __forceinline__ void copy_async16(void* shared, const void* global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(shared)), "l"(global) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void store_remote(uint32_t address, float a, float b, float c) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(address), "f"(a) : "memory");
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(address + 4), "f"(b) : "memory");
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(address + 8), "f"(c) : "memory");
}

// Where a thread stands: its unit, its rows and its column.
struct Post {
    int64_t b;
    int first_group, groups;  // of the unit
    int vector, column, columns;      // vector of the row; the same within the unit, of how many
    int lane, lanes, rank;
    int rows, each, extra;    // rows of this CTA: so many for each lane, and one more for the first few
    int64_t row0;
    bool active;
    __device__ __forceinline__ int rows_of(int l) const { return each + (l < extra ? 1 : 0); }
};
__device__ __forceinline__ Post post(const NormShape& s, const ResidentNorm& r, const int32_t* lengths, int V) {
    Post p;
    p.rank = blockIdx.x % (unsigned)r.cluster;
    const int64_t unit = blockIdx.x / (unsigned)r.cluster;
    p.b = unit / r.blocks;
    const int block = (int)(unit % r.blocks);
    p.first_group = block * r.groups;
    p.groups = min(r.groups, s.groups - p.first_group);
    p.columns = p.groups * s.width / V;
    p.lanes = blockDim.x / (unsigned)p.columns;
    p.lane = threadIdx.x / (unsigned)p.columns;
    p.column = threadIdx.x % (unsigned)p.columns;
    p.vector = p.first_group * s.width / V + p.column;
    p.active = p.lane < p.lanes;
    p.row0 = (int64_t)p.rank * r.rows;
    const int64_t left = positions_of(lengths, p.b, s.S) - p.row0;
    p.rows = (int)(left < 0 ? 0 : left < r.rows ? left : r.rows);
    p.each = p.rows / p.lanes;
    p.extra = p.rows % p.lanes;
    return p;
}

// Shared memory, behind the slots: results a group (float2), what the cluster's CTAs sent ([CTA][group] of three floats), and the room
// in which threads put their partial results side by side.
struct Room {
    uint4* slots;
    float2* result;
    float* sent;
    float2* side;
};
__device__ __forceinline__ Room room(const ResidentNorm& r, uint8_t* shared) {
    Room m;
    m.slots = reinterpret_cast<uint4*>(shared);
    m.result = reinterpret_cast<float2*>(shared + r.slot_bytes);
    m.sent = reinterpret_cast<float*>(m.result + r.groups);
    m.side = reinterpret_cast<float2*>(shared + r.side_offset);
    return m;
}

// A warp has this CTA's values of a group: its lanes write them into every CTA of the cluster.
__device__ __forceinline__ void send(const Room& m, const ResidentNorm& r, int rank, int group, float a, float b, float c) {
    const int lane = threadIdx.x & 31;
    if (lane < r.cluster) store_remote(ptx::map_to_cta(ptx::smem_u32(m.sent + (rank * r.groups + group) * 3), lane), a, b, c);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float element(const float2* v, int j) { return j % 2 ? v[j / 2].y : v[j / 2].x; }

// Mean and squared distances of a warp's entries, each of n values: the mean first, then the distances from it.  at(e) gives an entry's n
// and its (mean, squared distances).
template <typename At>
__device__ __forceinline__ Moments moments_of(int entries, At&& at) {
    const int lane = threadIdx.x & 31;
    float count = 0.0f, sum = 0.0f, m2 = 0.0f;
    for (int e = lane; e < entries; e += 32) {
        float n;
        const float2 v = at(e, &n);
        count += n;
        sum = fmaf(n, v.x, sum);
    }
    count = warp_sum(count);
    const float mean = count > 0.0f ? warp_sum(sum) / count : 0.0f;
    for (int e = lane; e < entries; e += 32) {
        float n;
        const float2 v = at(e, &n);
        m2 += n > 0.0f ? fmaf(n * (v.x - mean), v.x - mean, v.y) : 0.0f;
    }
    return Moments{count, mean, warp_sum(m2)};
}

template <typename IO, int ACT, int THREADS>
__global__ void __launch_bounds__(THREADS) resident_norm_kernel(NormShape s, ResidentNorm r, const uint4* x, const IO* gammas, const IO* betas,
                                                                const int32_t* lengths, uint4* y, float2* stats) {
    constexpr int V = NormIo<IO>::kVec, P = V / 2;
    extern __shared__ __align__(128) uint8_t shared[];
    const Room m = room(r, shared);
    ptx::grid_handover();
    __syncwarp();
    if (r.cluster > 1) ptx::cluster_arrive();
    const Post p = post(s, r, lengths, V);
    const int mine = p.active ? p.rows_of(p.lane) : 0, half = (mine + 1) / 2, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const uint4* from = x + (p.b * s.S + p.row0 + p.lane) * s.vectors + p.vector;
    const int64_t step = (int64_t)p.lanes * s.vectors;
    uint4* slot = m.slots + threadIdx.x;
    const int pitch = blockDim.x;
    for (int i = 0; i < half; ++i, from += step) copy_async16(slot + i * pitch, from);
    copies_commit();
    for (int i = half; i < mine; ++i, from += step) copy_async16(slot + i * pitch, from);
    copies_commit();

    RunningMoments<P> moments;
    auto add = [&](int i) {
        float2 f[P];
        NormIo<IO>::widen(slot[i * pitch], f);
        moments.add(f);
    };
    copies_wait<1>();
    for (int i = 0; i < half; ++i) add(i);
    copies_wait<0>();
    for (int i = half; i < mine; ++i) add(i);

    const bool whole = s.width % V == 0;                      // a vector lies in one group
    if (whole) {                                              // the columns of a vector have as many values each
        float mean = 0.0f, m2 = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j) mean += element(moments.mean, j);
        mean *= 1.0f / V;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float d = element(moments.mean, j) - mean;
            m2 += fmaf(moments.rows * d, d, element(moments.m2, j));
        }
        if (p.groups == 1) {                                  // every thread's: a warp's together
            const Moments t = moments_of(32, [&](int, float* n) { *n = moments.rows * V; return make_float2(mean, m2); });
            if ((threadIdx.x & 31) == 0) { m.side[2 * warp] = make_float2(t.mean, t.m2); m.side[2 * warp + 1].x = t.n; }
        } else {
            m.side[threadIdx.x] = make_float2(mean, m2);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) m.side[threadIdx.x * V + j] = make_float2(element(moments.mean, j), element(moments.m2, j));
    }
    __syncthreads();
    if (r.cluster > 1) ptx::cluster_wait();                   // the other CTAs have started: their shared memory may be written
    for (int g = warp; g < p.groups; g += warps) {
        Moments t;
        if (whole && p.groups == 1) {
            t = moments_of(warps, [&](int e, float* n) { *n = m.side[2 * e + 1].x; return m.side[2 * e]; });
        } else {
            // entries of a lane of rows: the group's vectors, or where they cross its border its elements
            const int per = whole ? 1 : V, width = whole ? s.width / V : s.width, pitch_of = p.columns * per;
            t = moments_of(min(p.lanes, p.rows) * width, [&](int e, float* n) {
                const int l = e / (unsigned)width;
                *n = (float)(p.rows_of(l) * (V / per));
                return m.side[l * pitch_of + g * width + e - l * width];
            });
        }
        if (r.cluster > 1) {
            send(m, r, p.rank, g, t.n, t.mean, t.m2);
        } else if ((threadIdx.x & 31) == 0) {
            const float2 out = make_float2(t.mean, rstd_of(t, s.eps));
            m.result[g] = out;
            if (stats) stats[p.b * s.groups + p.first_group + g] = out;
        }
    }
    __syncthreads();
    if (r.cluster > 1) {
        ptx::cluster_arrive();
        ptx::cluster_wait();
        for (int g = threadIdx.x; g < p.groups; g += blockDim.x) {
            Moments t{0.0f, 0.0f, 0.0f};
            for (int c = 0; c < r.cluster; ++c) {
                const float* at = m.sent + (c * r.groups + g) * 3;
                t = merge(t, Moments{at[0], at[1], at[2]});
            }
            const float2 out = make_float2(t.mean, rstd_of(t, s.eps));
            m.result[g] = out;
            if (stats && p.rank == 0) stats[p.b * s.groups + p.first_group + g] = out;
        }
        __syncthreads();
    }
    if (mine == 0) return;
    float2 mean[P], scale[P], beta[P];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int channel = (p.vector * V + j) / s.T;
        const float2 v = m.result[(p.column * V + j) / s.width];
        (&mean[j / 2].x)[j % 2] = v.x;
        (&scale[j / 2].x)[j % 2] = gammas ? NormIo<IO>::one(gammas, channel) * v.y : v.y;
        (&beta[j / 2].x)[j % 2] = betas ? NormIo<IO>::one(betas, channel) : 0.0f;
    }
    uint4* to = y + (p.b * s.S + p.row0 + p.lane) * s.vectors + p.vector;
    for (int i = 0; i < mine; ++i, to += step) {
        float2 f[P];
        NormIo<IO>::widen(slot[i * pitch], f);
#pragma unroll
        for (int j = 0; j < P; ++j) f[j] = activate<ACT>(fma2(sub2(f[j], mean[j]), scale[j], beta[j]));
        *to = NormIo<IO>::narrow(f);
    }
}

template <typename IO, int ACT, int THREADS>
__global__ void __launch_bounds__(THREADS) resident_gradient_kernel(NormShape s, ResidentNorm r, const uint4* x, const uint4* dy, const IO* gammas,
                                                                    const IO* betas, const int32_t* lengths, const float2* stats, uint4* dx, float2* parts) {
    constexpr int V = NormIo<IO>::kVec, P = V / 2;
    extern __shared__ __align__(128) uint8_t shared[];
    const Room m = room(r, shared);
    ptx::grid_handover();
    __syncwarp();
    if (r.cluster > 1) ptx::cluster_arrive();
    const Post p = post(s, r, lengths, V);
    const int mine = p.active ? p.rows_of(p.lane) : 0, half = (mine + 1) / 2, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t start = (p.b * s.S + p.row0 + p.lane) * s.vectors + p.vector, step = (int64_t)p.lanes * s.vectors;
    uint4* slot = m.slots + threadIdx.x;
    const int pitch = 2 * blockDim.x, second = blockDim.x;    // x and dy of a row are neighbours
    int64_t at = start;
    auto fetch = [&](int i) {
        copy_async16(slot + i * pitch, x + at);
        copy_async16(slot + i * pitch + second, dy + at);
        at += step;
    };
    for (int i = 0; i < half; ++i) fetch(i);
    copies_commit();
    for (int i = half; i < mine; ++i) fetch(i);
    copies_commit();
    float2 gamma[P], beta[P], mean[P], rstd[P];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int element = p.vector * V + j, channel = element / s.T;
        const float2 v = p.active ? stats[p.b * s.groups + element / s.width] : make_float2(0.0f, 0.0f);
        (&gamma[j / 2].x)[j % 2] = p.active && gammas ? NormIo<IO>::one(gammas, channel) : 1.0f;
        (&beta[j / 2].x)[j % 2] = p.active && betas ? NormIo<IO>::one(betas, channel) : 0.0f;
        (&mean[j / 2].x)[j % 2] = v.x;
        (&rstd[j / 2].x)[j % 2] = v.y;
    }
    float2 db[P] = {}, dg[P] = {}, xh[P], dz[P];
    auto both = [&](int i) {
        NormIo<IO>::widen(slot[i * pitch], xh);
        NormIo<IO>::widen(slot[i * pitch + second], dz);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            xh[j] = mul2(sub2(xh[j], mean[j]), rstd[j]);
            if (ACT != EQL_ACT_NONE) dz[j] = mul2(dz[j], slope<ACT>(fma2(xh[j], gamma[j], beta[j])));
        }
    };
    auto add = [&](int i) {
        both(i);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            db[j] = add2(db[j], dz[j]);
            dg[j] = fma2(dz[j], xh[j], dg[j]);
        }
    };
    copies_wait<1>();
    for (int i = 0; i < half; ++i) add(i);
    copies_wait<0>();
    for (int i = half; i < mine; ++i) add(i);

    // The thread's sums side by side: r.sums of them, of r.run neighbouring elements each (a channel's).
    float2 run = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        run.x += element(db, j);
        run.y += element(dg, j);
        if ((j + 1) % r.run == 0) {
            m.side[threadIdx.x * r.sums + j / r.run] = run;
            run = make_float2(0.0f, 0.0f);
        }
    }
    __syncthreads();
    // Channels: `share` lanes each, over the lanes of rows and the runs of the tuple.
    const int each = s.C / s.groups, channels = p.groups * each, runs = s.T / r.run, row = p.columns * r.sums;
    float2* sums = m.side + blockDim.x * r.sums;              // a channel's
    const int teams = blockDim.x / (unsigned)r.share, entries = min(p.lanes, p.rows) * runs, team = threadIdx.x / (unsigned)r.share;
    for (int c0 = 0; c0 < channels; c0 += teams) {
        const int c = c0 + team;
        float2 v = make_float2(0.0f, 0.0f);
        if (c < channels)
            for (int e = threadIdx.x - team * r.share; e < entries; e += r.share) {
                const int l = e / (unsigned)runs;
                v = add2(v, m.side[l * row + c * runs + e - l * runs]);
            }
        for (int d = r.share >> 1; d > 0; d >>= 1) {
            v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
            v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
        }
        if (c < channels && threadIdx.x == team * r.share) {
            sums[c] = v;
            parts[(p.b * r.cluster + p.rank) * s.C + p.first_group * each + c] = v;
        }
    }
    __syncthreads();
    if (r.cluster > 1) ptx::cluster_wait();
    const float count = (float)positions_of(lengths, p.b, s.S) * s.width, share = count > 0.0f ? 1.0f / count : 0.0f;
    for (int g = warp; g < p.groups; g += blockDim.x >> 5) {
        float2 v = make_float2(0.0f, 0.0f);
        for (int c = lane; c < each; c += 32) {
            const float w = gammas ? NormIo<IO>::one(gammas, (p.first_group + g) * each + c) : 1.0f;
            v = fma2(pair(w), sums[g * each + c], v);
        }
        v.x = warp_sum(v.x);
        v.y = warp_sum(v.y);
        if (r.cluster > 1) send(m, r, p.rank, g, v.x, v.y, 0.0f);
        else if (lane == 0) m.result[g] = make_float2(v.x * share, v.y * share);
    }
    __syncthreads();
    if (r.cluster > 1) {
        ptx::cluster_arrive();
        ptx::cluster_wait();
        for (int g = threadIdx.x; g < p.groups; g += blockDim.x) {
            float2 v = make_float2(0.0f, 0.0f);
            for (int c = 0; c < r.cluster; ++c) {
                const float* from = m.sent + (c * r.groups + g) * 3;
                v.x += from[0]; v.y += from[1];
            }
            m.result[g] = make_float2(v.x * share, v.y * share);
        }
        __syncthreads();
    }
    if (mine == 0) return;
    float2 off1[P], off2[P];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float2 v = m.result[(p.column * V + j) / s.width];
        (&off1[j / 2].x)[j % 2] = -v.x;
        (&off2[j / 2].x)[j % 2] = -v.y;
    }
    uint4* to = dx + start;
    for (int i = 0; i < mine; ++i, to += step) {
        both(i);
        float2 f[P];
#pragma unroll
        for (int j = 0; j < P; ++j) f[j] = mul2(rstd[j], fma2(xh[j], off2[j], fma2(gamma[j], dz[j], off1[j])));
        *to = NormIo<IO>::narrow(f);
    }
}

}  // namespace

constexpr int kFewThreads = 256, kManyForward = 1024, kManyBackward = 512;

ResidentNorm resident_norm_plan(const NormShape& s, eql_dtype_t dtype, bool backward) {
    ResidentNorm r{};
    const int V = dtype == EQL_FP32 ? 4 : 8;
    auto bytes = [&](int groups) { return (int64_t)groups * s.width / V * 16; };
    // Whole groups that begin and end with a vector, at least 128 bytes of a row; blocks of equal size that are whole 32-byte sectors
    // where there are such up to 512 bytes.
    int unit = 1;
    while (unit < s.groups && (int64_t)unit * s.width % V != 0) ++unit;
    r.groups = unit;
    while (r.groups < s.groups && bytes(r.groups) < 128) r.groups += unit;
    for (int g = r.groups; g <= s.groups && bytes(g) <= 512; g += unit)
        if (bytes(g) % 32 == 0 && s.groups % g == 0) { r.groups = g; break; }
    const int64_t columns = bytes(r.groups) / 16;
    if (columns > (backward ? kManyBackward : kManyForward)) return r;
    r.threads = columns <= kFewThreads ? kFewThreads : backward ? kManyBackward : kManyForward;
    r.blocks = (s.groups + r.groups - 1) / r.groups;
    r.run = s.T % V == 0 ? V : V % s.T == 0 ? s.T : 1;
    r.sums = V / r.run;
    const int channels = r.groups * (s.C / s.groups), lanes = (int)(r.threads / columns);
    const int side = backward ? r.threads * r.sums + channels : s.width % V == 0 ? r.threads : r.threads * V;
    for (r.cluster = 1; r.cluster <= kMaxCluster; r.cluster *= 2) {
        r.rows = (s.S + r.cluster - 1) / r.cluster;
        const int64_t slots = (r.rows + lanes - 1) / lanes, slot_bytes = slots * r.threads * 16 * (backward ? 2 : 1);
        r.side_offset = (int)align_up((size_t)r.groups * 8 + (size_t)r.cluster * r.groups * 12, 16);
        const int64_t all = slot_bytes + r.side_offset + side * 8;
        if (all <= kResidentShared) {
            r.slot_bytes = (int)slot_bytes;
            r.side_offset += r.slot_bytes;
            r.shared_bytes = (int)all;
            r.supported = true;
            // larger clusters until three CTAs fit an SM, and every SM has one or a thread has no more than four vectors
            if (all <= 74 * 1024 && (s.B * r.blocks * r.cluster >= kNumSMs || slots <= 4)) break;
        }
        if (r.cluster == kMaxCluster) break;
    }
    r.share = 1;
    while (r.share < 32 && r.share * 2 * channels <= r.threads) r.share *= 2;
    r.supported = r.supported && s.B * r.blocks * r.cluster <= INT32_MAX;
    return r;
}

template <typename Kernel, typename... Args>
static cudaError_t launch_resident(Kernel kernel, SmemLimitOnce& limit, const NormShape& s, const ResidentNorm& r, cudaStream_t stream, Args... args) {
    if (cudaError_t e = limit.ensure(kernel, kResidentShared); e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;      // see ptx::grid_dependency_wait
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)r.cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(s.B * r.blocks * r.cluster));
    cfg.blockDim = dim3(r.threads); cfg.dynamicSmemBytes = r.shared_bytes; cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = r.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, s, r, args...);
}

cudaError_t launch_resident_norm(const NormShape& s, const ResidentNorm& r, eql_dtype_t dtype, const void* x, const void* gamma, const void* beta,
                                 const int32_t* lengths, void* y, float* stats, cudaStream_t stream) {
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            static SmemLimitOnce limits[2];
            const bool few = r.threads == kFewThreads;
            return launch_resident(few ? resident_norm_kernel<IO, ACT, kFewThreads> : resident_norm_kernel<IO, ACT, kManyForward>, limits[few], s, r, stream, (const uint4*)x, (const IO*)gamma, (const IO*)beta,
                                   lengths, (uint4*)y, (float2*)stats);
        });
    });
}

cudaError_t launch_resident_gradient(const NormShape& s, const ResidentNorm& r, eql_dtype_t dtype, const void* x, const void* dy, const void* gamma,
                                     const void* beta, const int32_t* lengths, const float* stats, void* dx, float* parts, cudaStream_t stream) {
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            static SmemLimitOnce limits[2];
            const bool few = r.threads == kFewThreads;
            return launch_resident(few ? resident_gradient_kernel<IO, ACT, kFewThreads> : resident_gradient_kernel<IO, ACT, kManyBackward>, limits[few], s, r, stream, (const uint4*)x, (const uint4*)dy,
                                   (const IO*)gamma, (const IO*)beta, lengths, (const float2*)stats, (uint4*)dx, (float2*)parts);
        });
    });
}

}  // namespace eql
