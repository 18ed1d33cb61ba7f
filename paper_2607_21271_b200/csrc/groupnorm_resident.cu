// Group norm with an instance's groups resident in shared memory: x (and dy) are read once.
//
// A unit is a block of whole groups of one instance, at least 128 bytes of every row where there are as many.  It belongs to one CTA, or to a
// cluster whose CTAs hold a range of its rows each; what they have to tell each other is one triple (forward) or pair (backward) a
// group, written into every CTA's shared memory.  A thread stays with one 16-byte column, which it copies asynchronously into slots of its own: no
// barrier stands between copy and use, as many bytes are in flight as shared memory holds, and a slot that has been read for the last
// time takes a vector of the next instance at once.  What belongs to a column stays in registers for all instances that a CTA takes.
#include <algorithm>

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

// Where a thread stands: its block of groups, its column, its lane of rows, and its first instance.
struct Post {
    int64_t b, row0;
    int first_group, groups;  // of the block
    int vector, column, columns;      // vector of the row; the same within the block, of how many
    int lane, lanes, rank;
    Divisor by_lanes;
    bool active;
    __device__ __forceinline__ Post(const NormShape& s, const ResidentNorm& r, int V) {
        const unsigned unit = r.by_cluster(blockIdx.x), instance = r.by_blocks(unit), block = unit - instance * r.blocks;
        rank = blockIdx.x - unit * r.cluster;
        b = instance;
        first_group = block * r.groups;
        groups = min(r.groups, s.groups - first_group);
        Divisor by = r.columns;
        by_lanes = r.lanes;
        if (groups < r.groups) {                              // the last block, where it is a narrower one
            by = Divisor(groups * s.width / V);
            by_lanes = Divisor(by(blockDim.x));
        }
        columns = by.d;
        lanes = by_lanes.d;
        lane = by(threadIdx.x);
        column = threadIdx.x - lane * columns;
        vector = first_group * s.width / V + column;          // (V: a power of two)
        active = lane < lanes;
        row0 = (int64_t)rank * r.rows;
    }
    // this thread's first vector of an instance
    __device__ __forceinline__ int64_t at(const NormShape& s, int64_t instance) const { return (instance * s.S + row0 + lane) * s.vectors + vector; }
};
// The rows that a CTA has of an instance, dealt to its lanes: so many each, one more for the first few.
struct Rows {
    int all, each, extra;
    __device__ __forceinline__ Rows(const NormShape& s, const ResidentNorm& r, const Post& p, const int32_t* lengths, int64_t b) {
        const int64_t left = b < s.B ? positions_of(lengths, b, s.S) - p.row0 : 0;
        all = (int)(left < 0 ? 0 : left < r.rows ? left : r.rows);
        each = p.by_lanes(all);
        extra = all - each * p.lanes;
    }
    __device__ __forceinline__ int of(int lane) const { return each + (lane < extra ? 1 : 0); }
};
// Shared memory, behind the slots: results a group (float2), what the cluster's CTAs sent (for this instance and the one before:
// [2][CTA][group] of three floats), and the room in which threads put their partial results side by side.
struct Room {
    uint4* slots;
    float2* result;
    float* sent;
    float2* side;
    __device__ __forceinline__ Room(const ResidentNorm& r, uint8_t* shared) {
        slots = reinterpret_cast<uint4*>(shared);
        result = reinterpret_cast<float2*>(shared + r.slot_bytes);
        sent = reinterpret_cast<float*>(result + r.groups);
        side = reinterpret_cast<float2*>(shared + r.side_offset);
    }
    __device__ __forceinline__ float* from(const ResidentNorm& r, int round, int rank, int group) const {
        return sent + (((round & 1) * r.cluster + rank) * r.groups + group) * 3;
    }
    // A warp has this CTA's values of a group: its lanes write them into every CTA of the cluster.  (Into the half that the other
    // CTAs read an instance ago: they have all passed the barrier of the one in between.)
    __device__ __forceinline__ void send(const ResidentNorm& r, int round, int rank, int group, float a, float b, float c) const {
        const int lane = threadIdx.x & 31;
        if (lane < r.cluster) store_remote(ptx::map_to_cta(ptx::smem_u32(from(r, round, rank, group)), lane), a, b, c);
    }
};

// use(i) for the `mine` slots of one instance, and copy(i) into the `count` slots of the next one, each slot as soon as it has been used;
// the copies in two groups, so that the first half can be used while the second is on its way.
template <typename Use, typename Copy>
__device__ __forceinline__ void refill(int mine, int count, Use&& use, Copy&& copy) {
    const int half = (count + 1) / 2;
    int i = 0;
#pragma unroll 2
    for (; i < half; ++i) {
        if (i < mine) use(i);
        copy(i);
    }
    copies_commit();
#pragma unroll 2
    for (; i < count; ++i) {
        if (i < mine) use(i);
        copy(i);
    }
    copies_commit();
#pragma unroll 2
    for (; i < mine; ++i) use(i);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float element(const float2* v, int j) { return j % 2 ? v[j / 2].y : v[j / 2].x; }

// Mean and squared distances of a warp's entries, each of n values, `count` in all.  at(e) gives an entry's n and its (mean, squared
// distances); no entry is of no values.  The entries' means are taken relative to the average of the lanes' first ones, which a single far
// value moves by no more than a 32nd of what it moves its own entry's mean (or by its share, of fewer entries).
template <typename At>
__device__ __forceinline__ Moments moments_of(float count, int entries, At&& at) {
    const int lane = threadIdx.x & 31;
    float sum = 0.0f, m2 = 0.0f, n = 0.0f;
    float2 v = make_float2(0.0f, 0.0f);
    if (lane < entries) v = at(lane, &n);
    const float middle = entries > 0 ? __fdividef(warp_sum(v.x), (float)min(entries, 32)) : 0.0f;
    for (int e = lane; e < entries;) {
        const float d = v.x - middle;
        sum = fmaf(n, d, sum);
        m2 += fmaf(n * d, d, v.y);
        e += 32;
        if (e < entries) v = at(e, &n);
    }
    sum = warp_sum(sum);
    m2 = warp_sum(m2);
    const float mean = count > 0.0f ? __fdividef(sum, count) : 0.0f;
    m2 -= sum * mean;
    return Moments{count, middle + mean, m2 < 0.0f ? 0.0f : m2};
}

// The groups of a vector's runs, relative to its first element's: three bits each.
template <typename R>
__device__ __forceinline__ unsigned group_steps(const NormShape& s, int in_group) {
    unsigned steps = 0;
    if (R::kEntries > 1) R::each(0, in_group, s.width, [&](int e, int step) { steps |= (unsigned)step << (3 * e); });
    return steps;
}
template <typename R, typename Set>
__device__ __forceinline__ void each_group(unsigned steps, const float2* first, Set&& set) {
#pragma unroll
    for (int e = 0; e < R::kEntries; ++e) set(e, first[steps >> (3 * e) & 7u]);
}
// Gamma and beta of a thread's column.  What is read outside the slots is asked for before their copies, behind which it would wait for
// thousands of cycles, and looked at after them.
template <typename IO, typename R>
struct Parameters {
    IO gamma[R::kEntries], beta[R::kEntries];
    __device__ __forceinline__ void load(const NormShape& s, const ResidentNorm& r, const Post& p, const IO* gammas, const IO* betas) {
        const int first = r.tuple(p.column * NormIo<IO>::kVec), block = p.first_group * (s.C / s.groups);
        R::each(first, p.column * NormIo<IO>::kVec - first * s.T, s.T, [&](int e, int channel) {
            if (p.active && gammas) gamma[e] = gammas[block + channel];
            if (p.active && betas) beta[e] = betas[block + channel];
        });
    }
    __device__ __forceinline__ void get(const Post& p, const IO* gammas, const IO* betas, R* g, R* b) const {
#pragma unroll
        for (int e = 0; e < R::kEntries; ++e) {
            g->set(e, p.active && gammas ? NormIo<IO>::one(gamma, e) : 1.0f);
            b->set(e, p.active && betas ? NormIo<IO>::one(beta, e) : 0.0f);
        }
    }
};

// N: see Runs.
template <typename IO, int ACT, int N, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) resident_norm_kernel(NormShape s, ResidentNorm r, const uint4* x, const IO* gammas, const IO* betas,
                                                                      const int32_t* lengths, uint4* y, float2* stats) {
    constexpr int V = NormIo<IO>::kVec, P = V / 2;
    extern __shared__ __align__(128) uint8_t shared[];
    const Room m(r, shared);
    ptx::grid_handover();
    __syncwarp();
    if (r.cluster > 1) ptx::cluster_arrive();
    const Post p(s, r, V);
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, pitch = blockDim.x;
    const int64_t step = (int64_t)p.lanes * s.vectors;
    uint4* slot = m.slots + threadIdx.x;
    Rows rows(s, r, p, lengths, p.b);
    int mine = p.active ? rows.of(p.lane) : 0;
    Parameters<IO, Runs<N, P>> raw;
    raw.load(s, r, p, gammas, betas);
    {
        const uint4* from = x + p.at(s, p.b);
        refill(0, mine, [](int) {}, [&](int i) { copy_async16(slot + i * pitch, from); from += step; });
    }
    const bool whole = N == 1 || s.width % V == 0;            // a vector lies in one group
    const int group = r.width(p.column * V);                  // of the block, that of the first element
    const unsigned steps = group_steps<Runs<N, P>>(s, p.column * V - group * s.width);
    int round = 0;
    for (int64_t b = p.b; b < s.B; b += r.instances, ++round) {
        RunningMoments<P> moments;
        auto add = [&](int i) {
            float2 f[P];
            NormIo<IO>::widen(slot[i * pitch], f);
            moments.add(f);
        };
        const int half = (mine + 1) / 2;
        copies_wait<1>();
#pragma unroll 2
        for (int i = 0; i < half; ++i) add(i);
        copies_wait<0>();
#pragma unroll 2
        for (int i = half; i < mine; ++i) add(i);
        // The columns of `pairs` pairs from `first` on, which have as many values each.
        auto together = [&](int first, int pairs) {
            float2 sum = moments.mean[first], squares = moments.m2[first];
#pragma unroll
            for (int j = 1; j < pairs; ++j) sum = add2(sum, moments.mean[first + j]);
            const float mean = (sum.x + sum.y) * (0.5f / pairs);
            float2 off = sub2(moments.mean[first], pair(mean)), around = mul2(off, off);
#pragma unroll
            for (int j = 1; j < pairs; ++j) {
                off = sub2(moments.mean[first + j], pair(mean));
                around = fma2(off, off, around);
                squares = add2(squares, moments.m2[first + j]);
            }
            squares = fma2(around, pair(moments.rows), squares);
            return make_float2(mean, squares.x + squares.y);
        };
        if (whole) {
            const float2 t = together(0, P);
            const float mean = t.x, m2 = t.y;
            if (p.groups == 1) {                              // every thread's: a warp's together
                const float n = moments.rows * V, all = warp_sum(n), middle = all > 0.0f ? __fdividef(warp_sum(n * mean), all) : 0.0f;
                const float around_all = warp_sum(fmaf(n * (mean - middle), mean - middle, m2));
                if ((threadIdx.x & 31) == 0) { m.side[2 * warp] = make_float2(middle, around_all); m.side[2 * warp + 1].x = all; }
            } else {
                m.side[threadIdx.x] = t;
            }
        } else if (N == 2 && P > 2) {
            m.side[threadIdx.x * 2] = together(0, P / 2);
            m.side[threadIdx.x * 2 + 1] = together(P / 2, P / 2);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) m.side[threadIdx.x * V + j] = make_float2(element(moments.mean, j), element(moments.m2, j));
        }
        __syncthreads();
        if (r.cluster > 1 && round == 0) ptx::cluster_wait(); // the other CTAs have started: their shared memory may be written
        for (int g = warp; g < p.groups; g += warps) {
            Moments t;
            const float count = (float)rows.all * s.width;
            if (whole && p.groups == 1) {
                // the warps that have rows: the threads that do are the first ones, lane by lane.  (An idle warp's mean of 0 in the entries'
                // average costs far means their digits: 640 floats about 1000 with a spread of 1, three warps of eight idle, gave y up to 0.03 off.)
                t = moments_of(count, (min(p.lanes, rows.all) * p.columns + 31) >> 5, [&](int e, float* n) { *n = m.side[2 * e + 1].x; return m.side[2 * e]; });
            } else {
                // entries of a lane of rows: the group's vectors, or where they cross its border its runs
                const int per = whole ? 1 : Runs<N, P>::kEntries, row = p.columns * per;
                const float more = (float)((rows.each + 1) * (V / per)), fewer = (float)(rows.each * (V / per));
                t = moments_of(count, min(p.lanes, rows.all) * (int)r.entry.d, [&](int e, float* n) {
                    const int l = r.entry(e);
                    *n = l < rows.extra ? more : fewer;
                    return m.side[l * row + (g - l) * (int)r.entry.d + e];
                });
            }
            if (r.cluster > 1) {
                m.send(r, round, p.rank, g, t.n, t.mean, t.m2);
            } else if ((threadIdx.x & 31) == 0) {
                const float2 out = make_float2(t.mean, rstd_of(t, s.eps));
                m.result[g] = out;
                if (stats) stats[b * s.groups + p.first_group + g] = out;
            }
        }
        __syncthreads();
        if (r.cluster > 1) {
            ptx::cluster_arrive();
            ptx::cluster_wait();
            for (int g = threadIdx.x; g < p.groups; g += blockDim.x) {
                // relative to the first CTA's mean, which is none of theirs where it has no rows
                const float middle = m.from(r, round, 0, g)[1];
                float n = 0.0f, sum = 0.0f, m2 = 0.0f;
                for (int c = 0; c < r.cluster; ++c) {
                    const float* at = m.from(r, round, c, g);
                    if (!(at[0] > 0.0f)) continue;
                    const float d = at[1] - middle;
                    n += at[0];
                    sum = fmaf(at[0], d, sum);
                    m2 += fmaf(at[0] * d, d, at[2]);
                }
                const float off = n > 0.0f ? __fdividef(sum, n) : 0.0f;
                m2 -= sum * off;
                const Moments t{n, middle + off, m2 < 0.0f ? 0.0f : m2};
                const float2 out = make_float2(t.mean, rstd_of(t, s.eps));
                m.result[g] = out;
                if (stats && p.rank == 0) stats[b * s.groups + p.first_group + g] = out;
            }
            __syncthreads();
        }
        Runs<N, P> mean, scale, gamma, beta;
        raw.get(p, gammas, betas, &gamma, &beta);
        each_group<Runs<N, P>>(steps, m.result + group, [&](int e, float2 v) {
            mean.set(e, v.x);
            scale.set(e, v.y);
        });
#pragma unroll
        for (int j = 0; j < N; ++j) scale.v[j] = mul2(scale.v[j], gamma.v[j]);
        // every slot, once used, takes the next instance's vector
        const Rows next = lengths || b + r.instances >= s.B ? Rows(s, r, p, lengths, b + r.instances) : rows;
        const int count = p.active ? next.of(p.lane) : 0;
        uint4* to = y + p.at(s, b);
        const uint4* from = x + p.at(s, b + r.instances);
        auto apply = [&](int i) {
            float2 f[P];
            NormIo<IO>::widen(slot[i * pitch], f);
#pragma unroll
            for (int j = 0; j < P; ++j) f[j] = activate<ACT, (N < P)>(fma2(sub2(f[j], mean.of(j)), scale.of(j), beta.of(j)));
            *to = NormIo<IO>::narrow(f);
            to += step;
        };
        refill(mine, count, apply, [&](int i) { copy_async16(slot + i * pitch, from); from += step; });
        rows = next;
        mine = count;
    }
}

template <typename IO, int ACT, int N, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) resident_gradient_kernel(NormShape s, ResidentNorm r, const uint4* x, const uint4* dy, const IO* gammas,
                                                                          const IO* betas, const int32_t* lengths, const float2* stats, uint4* dx,
                                                                          float2* parts) {
    constexpr int V = NormIo<IO>::kVec, P = V / 2;
    extern __shared__ __align__(128) uint8_t shared[];
    const Room m(r, shared);
    ptx::grid_handover();
    __syncwarp();
    if (r.cluster > 1) ptx::cluster_arrive();
    const Post p(s, r, V);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t step = (int64_t)p.lanes * s.vectors;
    uint4* slot = m.slots + threadIdx.x;
    const int pitch = 2 * blockDim.x, second = blockDim.x;    // x and dy of a row are neighbours
    Rows rows(s, r, p, lengths, p.b);
    int mine = p.active ? rows.of(p.lane) : 0;
    const int group = r.width(p.column * V);                  // of the block, that of the first element
    const unsigned steps = group_steps<Runs<N, P>>(s, p.column * V - group * s.width);
    const int each = s.C / s.groups, channels = p.groups * each, row = p.columns * r.sums;
    Parameters<IO, Runs<N, P>> raw;
    raw.load(s, r, p, gammas, betas);
    float2 saved[Runs<N, P>::kEntries];                       // mean and rstd of the column's groups
    each_group<Runs<N, P>>(steps, stats + p.b * s.groups + p.first_group + group, [&](int e, float2 v) { saved[e] = v; });
    {
        const uint4 *from_x = x + p.at(s, p.b), *from_dy = dy + p.at(s, p.b);
        refill(0, mine, [](int) {}, [&](int i) {
            copy_async16(slot + i * pitch, from_x);
            copy_async16(slot + i * pitch + second, from_dy);
            from_x += step;
            from_dy += step;
        });
    }
    Runs<N, P> gamma, beta;
    raw.get(p, gammas, betas, &gamma, &beta);
    const bool whole = N == 1 || s.width % V == 0;            // a vector lies in one group
    float2* total = m.side + blockDim.x * (r.sums + (whole ? 1 : Runs<N, P>::kEntries));      // a channel's sums over all instances so far
    const int teams = blockDim.x / (unsigned)r.share, team = threadIdx.x / (unsigned)r.share;
    for (int c = threadIdx.x; c < channels; c += blockDim.x) total[c] = make_float2(0.0f, 0.0f);
    int round = 0;
    for (int64_t b = p.b; b < s.B; b += r.instances, ++round) {
        // z = (x - mean) * (rstd * gamma) + beta;  rstd comes to the sums of dz * (x - mean) at the end
        Runs<N, P> mean, scale, rstd;
#pragma unroll
        for (int e = 0; e < Runs<N, P>::kEntries; ++e) {
            mean.set(e, saved[e].x);
            rstd.set(e, saved[e].y);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) scale.v[j] = mul2(rstd.v[j], gamma.v[j]);
        float2 db[P] = {}, dg[P] = {}, xc[P], dz[P];
        // A float dz takes the place of dy, and is there the second time; in 16 bits it would lose, and is computed again.
        constexpr bool kKeep = sizeof(IO) == 4 && ACT != EQL_ACT_NONE;
        auto both = [&](int i, bool again) {
            NormIo<IO>::widen(slot[i * pitch], xc);
            NormIo<IO>::widen(slot[i * pitch + second], dz);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                xc[j] = sub2(xc[j], mean.of(j));
                if (ACT != EQL_ACT_NONE && !(kKeep && again)) dz[j] = mul2(dz[j], slope<ACT, (N < P)>(fma2(xc[j], scale.of(j), beta.of(j))));
            }
        };
        auto add = [&](int i) {
            both(i, false);
            if (kKeep) slot[i * pitch + second] = NormIo<IO>::narrow(dz);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const int k = N == 1 ? j % 2 : j * N / P;     // (two chains are enough where one number comes out)
                db[k] = add2(db[k], dz[j]);
                dg[k] = fma2(dz[j], xc[j], dg[k]);
            }
        };
        const int half = (mine + 1) / 2;
        copies_wait<1>();
#pragma unroll 2
        for (int i = 0; i < half; ++i) add(i);
        copies_wait<0>();
#pragma unroll 2
        for (int i = half; i < mine; ++i) add(i);

        // The thread's sums side by side: r.sums of them, of r.run neighbouring elements each (a channel's); and times gamma, for the
        // groups, of its vector or where groups cross that of its runs.
        float2* weighted = m.side + blockDim.x * r.sums;
        if (N == 1) {
            db[0] = add2(db[0], db[1]);
            dg[0] = mul2(add2(dg[0], dg[1]), rstd.v[0]);
            const float2 v = make_float2(db[0].x + db[0].y, dg[0].x + dg[0].y);
            m.side[threadIdx.x] = v;
            weighted[threadIdx.x] = mul2(v, gamma.v[0]);
        } else {
            float2 all1 = pair(0.0f), all2 = pair(0.0f);
            float2 *to = m.side + threadIdx.x * r.sums, *each_weighted = weighted + threadIdx.x * Runs<N, P>::kEntries;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                dg[j] = mul2(dg[j], rstd.v[j]);
                const float2 w1 = mul2(db[j], gamma.v[j]), w2 = mul2(dg[j], gamma.v[j]);
                if (r.sums <= N) {
                    to[j] = make_float2(db[j].x + db[j].y, dg[j].x + dg[j].y);
                } else {                                      // (each half of a pair is a channel's)
                    to[2 * j] = make_float2(db[j].x, dg[j].x);
                    to[2 * j + 1] = make_float2(db[j].y, dg[j].y);
                }
                if (whole) {
                    all1 = add2(all1, w1);
                    all2 = add2(all2, w2);
                } else if (N < P) {
                    each_weighted[j] = make_float2(w1.x + w1.y, w2.x + w2.y);
                } else {
                    each_weighted[2 * j] = make_float2(w1.x, w2.x);
                    each_weighted[2 * j + 1] = make_float2(w1.y, w2.y);
                }
            }
            if (whole) weighted[threadIdx.x] = make_float2(all1.x + all1.y, all2.x + all2.y);
        }
        __syncthreads();
        if (r.cluster > 1 && round == 0) ptx::cluster_wait();
        const float count = (float)positions_of(lengths, b, s.S) * s.width, share = count > 0.0f ? __fdividef(1.0f, count) : 0.0f;
        const int row_lanes = min(p.lanes, rows.all), per = whole ? 1 : Runs<N, P>::kEntries;
        // Channels: `share` lanes each, over the lanes of rows and the runs of the tuple.
        auto add_channels = [&]() {
            const int entries = row_lanes * (int)r.runs.d;
            for (int c0 = 0; c0 < channels; c0 += teams) {
                const int c = c0 + team;
                float2 v = make_float2(0.0f, 0.0f);
                if (c < channels)
                    for (int e = threadIdx.x - team * r.share; e < entries; e += r.share) {
                        const int l = r.runs(e);
                        v = add2(v, m.side[l * row + (c - l) * (int)r.runs.d + e]);
                    }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1)
                    if (d < r.share) {
                        v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
                        v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
                    }
                if (c < channels && threadIdx.x == team * r.share) total[c] = add2(total[c], v);
            }
        };
        for (int g = warp; g < p.groups; g += blockDim.x >> 5) {
            const int width = (int)r.entry.d;                 // entries of the group in a lane of rows
            float2 v = make_float2(0.0f, 0.0f);
            for (int e = lane; e < row_lanes * width; e += 32) {
                const int l = r.entry(e);
                v = add2(v, weighted[l * p.columns * per + (g - l) * width + e]);
            }
            v.x = warp_sum(v.x);
            v.y = warp_sum(v.y);
            if (r.cluster > 1) m.send(r, round, p.rank, g, v.x, v.y, 0.0f);
            else if (lane == 0) m.result[g] = make_float2(v.x * share, v.y * share);
        }
        if (r.cluster == 1) add_channels();
        __syncthreads();
        if (r.cluster > 1) ptx::cluster_arrive();
        if (r.cluster > 1) add_channels();                    // while the other CTAs come
        if (r.cluster > 1) {
            __syncwarp();
            ptx::cluster_wait();
            for (int g = threadIdx.x; g < p.groups; g += blockDim.x) {
                float2 v = make_float2(0.0f, 0.0f);
                for (int c = 0; c < r.cluster; ++c) {
                    const float* from = m.from(r, round, c, g);
                    v.x += from[0]; v.y += from[1];
                }
                m.result[g] = make_float2(v.x * share, v.y * share);
            }
            __syncthreads();
        }
        // dx = dz * (rstd * gamma) - (x - mean) * (rstd * rstd * second) - rstd * first
        Runs<N, P> off1, off2;
        each_group<Runs<N, P>>(steps, m.result + group, [&](int e, float2 v) {
            off1.set(e, -v.x);
            off2.set(e, -v.y);
        });
#pragma unroll
        for (int j = 0; j < N; ++j) {
            off1.v[j] = mul2(off1.v[j], rstd.v[j]);
            off2.v[j] = mul2(mul2(off2.v[j], rstd.v[j]), rstd.v[j]);
        }
        const Rows next = lengths || b + r.instances >= s.B ? Rows(s, r, p, lengths, b + r.instances) : rows;
        const int count_next = p.active ? next.of(p.lane) : 0;
        if (b + r.instances < s.B)
            each_group<Runs<N, P>>(steps, stats + (b + r.instances) * s.groups + p.first_group + group, [&](int e, float2 v) { saved[e] = v; });
        uint4* to = dx + p.at(s, b);
        const uint4 *from_x = x + p.at(s, b + r.instances), *from_dy = dy + p.at(s, b + r.instances);
        auto apply = [&](int i) {
            both(i, true);
            float2 f[P];
#pragma unroll
            for (int j = 0; j < P; ++j) f[j] = fma2(xc[j], off2.of(j), fma2(dz[j], scale.of(j), off1.of(j)));
            *to = NormIo<IO>::narrow(f);
            to += step;
        };
        refill(mine, count_next, apply, [&](int i) {
            copy_async16(slot + i * pitch, from_x);
            copy_async16(slot + i * pitch + second, from_dy);
            from_x += step;
            from_dy += step;
        });
        rows = next;
        mine = count_next;
    }
    float2* out = parts + (p.b * r.cluster + p.rank) * s.C + p.first_group * each;
    for (int c0 = 0; c0 < channels; c0 += teams)               // (each by the thread that added it up)
        if (c0 + team < channels && threadIdx.x == team * r.share) out[c0 + team] = total[c0 + team];
}

}  // namespace

constexpr int kFewThreads = 256, kManyForward = 1024, kManyBackward = 512;
// CTAs of 256 threads to an SM, by the registers that the kernels then may use.  (Backward, with two instead of three and two rows of a
// thread side by side: 128 x 3136 x 384 bfloat16, forward and backward, 533 -> 519 us.)
constexpr int forward_ctas(int n, int P) { return n < P ? 4 : 3; }
constexpr int kGradientCtas = 2;

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
    r.form = r.threads == kFewThreads ? runs_of(s.T, V) : V / 2;              // (with many threads there is the general form only)
    r.blocks = (s.groups + r.groups - 1) / r.groups;
    r.run = std::min(run_length(s.T, V), V / r.form);         // (a thread of form N keeps N pairs of sums at least)
    r.sums = V / r.run;
    r.tuple = Divisor(s.T);
    r.width = Divisor(s.width);
    const int per = s.width % V == 0 ? 1 : entries_of(r.form, V / 2);         // entries of a vector
    r.entry = Divisor(s.width * per / V);
    r.runs = Divisor(s.T / r.run);
    r.columns = Divisor((unsigned)columns);
    r.lanes = Divisor((unsigned)(r.threads / columns));
    r.by_blocks = WideDivisor(r.blocks);
    const int channels = r.groups * (s.C / s.groups), lanes = (int)(r.threads / columns);
    const int side = backward ? r.threads * (r.sums + per) + channels : r.threads * per;
    for (r.cluster = 1; r.cluster <= kMaxCluster; r.cluster *= 2) {
        r.rows = (s.S + r.cluster - 1) / r.cluster;
        const int64_t slots = (r.rows + lanes - 1) / lanes, slot_bytes = slots * r.threads * 16 * (backward ? 2 : 1);
        r.side_offset = (int)align_up((size_t)r.groups * 8 + (size_t)r.cluster * r.groups * 24, 16);
        const int64_t all = slot_bytes + r.side_offset + side * 8;
        if (all <= kResidentShared) {
            r.slot_bytes = (int)slot_bytes;
            r.side_offset += r.slot_bytes;
            r.shared_bytes = (int)all;
            r.supported = true;
            // One CTA where two of them fit an SM; else larger clusters until three do, and every SM has one or a thread has no more than
            // four vectors.  (Backward, one CTA of 83 KB / clusters of two with 42 KB: 128 x 197 x 768 bfloat16 38 / 49 us.)
            if (all <= (r.cluster == 1 ? 112 : 74) * 1024 && (s.B * r.blocks * r.cluster >= kNumSMs || slots <= 4)) break;
        }
        if (r.cluster == kMaxCluster) break;
    }
    if (!r.supported) return r;
    r.by_cluster = WideDivisor(r.cluster);
    r.share = 1;
    while (r.share < 32 && r.share * 2 * channels <= r.threads) r.share *= 2;
    // One CTA after the other takes a block's instances, as many side by side as are resident together, and all about the same number.
    // (A cluster takes one: how many of them are resident depends on the SMs that the device has in each of its parts.)
    int64_t together = 228 * 1024 / (r.shared_bytes + 1024), most = backward ? kGradientCtas : forward_ctas(r.form, V / 2);
    if (r.threads != kFewThreads) most = 1;
    if (together > most) together = most;
    together = together * kNumSMs / (r.blocks * r.cluster);
    if (together < 1) together = 1;
    r.instances = (int)s.B;
    if (r.cluster == 1 && together < s.B) {
        const int64_t rounds = (s.B + together - 1) / together;
        r.instances = (int)((s.B + rounds - 1) / rounds);
    }
    r.supported = (int64_t)r.instances * r.blocks * r.cluster <= INT32_MAX;
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
    cfg.gridDim = dim3((unsigned)((int64_t)r.instances * r.blocks * r.cluster));
    cfg.blockDim = dim3(r.threads); cfg.dynamicSmemBytes = r.shared_bytes; cfg.stream = stream;
    cfg.attrs = attr; cfg.numAttrs = r.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, s, r, args...);
}

cudaError_t launch_resident_norm(const NormShape& s, const ResidentNorm& r, eql_dtype_t dtype, const void* x, const void* gamma, const void* beta,
                                 const int32_t* lengths, void* y, float* stats, cudaStream_t stream) {
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        constexpr int V = NormIo<IO>::kVec, P = V / 2;
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            static SmemLimitOnce limits[4];
            auto launch = [&](auto kernel, SmemLimitOnce& limit) {
                return launch_resident(kernel, limit, s, r, stream, (const uint4*)x, (const IO*)gamma, (const IO*)beta, lengths, (uint4*)y, (float2*)stats);
            };
            if (r.threads != kFewThreads) return launch(resident_norm_kernel<IO, ACT, P, kManyForward, 1>, limits[0]);
            if (r.form == 1) return launch(resident_norm_kernel<IO, ACT, 1, kFewThreads, forward_ctas(1, P)>, limits[1]);
            if (r.form < P) return launch(resident_norm_kernel<IO, ACT, 2, kFewThreads, forward_ctas(2, P)>, limits[2]);
            return launch(resident_norm_kernel<IO, ACT, P, kFewThreads, forward_ctas(P, P)>, limits[3]);
        });
    });
}

cudaError_t launch_resident_gradient(const NormShape& s, const ResidentNorm& r, eql_dtype_t dtype, const void* x, const void* dy, const void* gamma,
                                     const void* beta, const int32_t* lengths, const float* stats, void* dx, float* parts, cudaStream_t stream) {
    return dispatch_io(dtype, [&](auto io) {
        using IO = decltype(io);
        constexpr int V = NormIo<IO>::kVec, P = V / 2;
        return dispatch_act(s.act, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            static SmemLimitOnce limits[4];
            auto launch = [&](auto kernel, SmemLimitOnce& limit) {
                return launch_resident(kernel, limit, s, r, stream, (const uint4*)x, (const uint4*)dy, (const IO*)gamma, (const IO*)beta, lengths,
                                       (const float2*)stats, (uint4*)dx, (float2*)parts);
            };
            if (r.threads != kFewThreads) return launch(resident_gradient_kernel<IO, ACT, P, kManyBackward, 1>, limits[0]);
            if (r.form == 1) return launch(resident_gradient_kernel<IO, ACT, 1, kFewThreads, kGradientCtas>, limits[1]);
            if (r.form < P) return launch(resident_gradient_kernel<IO, ACT, 2, kFewThreads, kGradientCtas>, limits[2]);
            return launch(resident_gradient_kernel<IO, ACT, P, kFewThreads, kGradientCtas>, limits[3]);
        });
    });
}

}  // namespace eql
