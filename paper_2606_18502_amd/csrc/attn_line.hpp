// How the paged attention kernels share out their work, and join what is split.
//
// A unit is (sequence, ROWS rows of a KV head's group, HG KV heads); its work is
// its number of key steps.  The lengths are the device's, so the cut is made there.
// Much work: the units lie on one line in the order sequence, heads, row tile (a head's tiles
// read the same keys), each with its steps and `extra` more for its beginning and end,
// and the workgroups cut the line into equal ranges, whatever the sequences' lengths: a
// range covers whole units and parts of at most two.  Little work (fewer than CELL steps
// for every workgroup): a unit is cut into cells of about CELL steps, one workgroup each; a
// shorter one is not worth its join.
// The parts of a unit are joined by the workgroup that stores the last of
// them, found by a ticket; many parts in two rounds, the first over runs of parts.
//
// No fences: parts are stored and loaded with relaxed accesses at agent scope
// (through to where all XCDs meet), a wave waits for the acknowledgement of its
// stores before the workgroup takes its ticket, and the last one loads only
// after its ticket has returned.
#pragma once

#include "attn_common.hpp"

namespace specfp8 {

namespace {

constexpr int kJoin = 16;                                    // parts that one workgroup joins at a time

template <int THREADS>
struct LineShared {
    int64_t scan[THREADS / 64], found[2];
    int window[3][32];                                       // first row, rows and tokens of some sequences
    int is_last;
};

template <int THREADS, int ROWS, int STEP, int CELL>
struct Line {
    int64_t total, hi, pos, base;
    int ng, wg, b, window_at, nhg;
    int extra;                                               // < 0: cells
    // the current segment: steps s_in .. s_in + count of a unit of `steps`, part `me` of `parts` from workgroup w0 on
    int first, n, L, steps, rt, hg, s_in, count, w0, parts, me;

    // what a unit takes of the line
    static __device__ __forceinline__ int length(int steps, int extra) { return extra < 0 ? max((steps + 1) / CELL, 1) : steps + extra; }
    static __device__ __forceinline__ int64_t units(const PagedArgs& a, int n, int nhg) {
        return (((int64_t)n * (a.Hq / a.H) + ROWS - 1) / ROWS) * nhg;
    }
    struct Sequence {
        int first, n, L;
        __device__ __forceinline__ Sequence(const PagedArgs& a, int b) {
            rows_of(a.cu_q, a.T, a.B, b, &first, &n);
            L = min(max(a.kv_lens[b], 0), a.max_len);
        }
    };
    static __device__ __forceinline__ int64_t cost_of(const PagedArgs& a, const Sequence& s, int nhg, int extra) {
        return units(a, s.n, nhg) * length(max((s.L + STEP - 1) / STEP, 1), extra);
    }
    static __device__ __forceinline__ int64_t sum_before(int64_t mine, int64_t* scan, int64_t* sum) {
        const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
        int64_t upto = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 63) scan[w] = upto;
        __syncthreads();
        int64_t before = 0, all = 0;
        for (int x = 0; x < THREADS / 64; ++x) {
            if (x < w) before += scan[x];
            all += scan[x];
        }
        *sum = all;
        return before + upto - mine;
    }

    // This workgroup's range; false if it has none.  Called by all threads.
    __device__ __forceinline__ bool begin(const PagedArgs& a, LineShared<THREADS>& sh, int heads, int groups, int extra_) {
        const int tid = threadIdx.x;
        nhg = (a.H + heads - 1) / heads;
        const int per = (a.B + THREADS - 1) / THREADS;
        const Sequence own(a, min(tid * per, a.B - 1));      // (the first of this thread's; mostly the only one)
        const auto sum_here = [&](int how) {
            int64_t v = tid * per < a.B ? cost_of(a, own, nhg, how) : 0;
            for (int x = 1; x < per && tid * per + x < a.B; ++x) v += cost_of(a, Sequence(a, tid * per + x), nhg, how);
            return v;
        };
        extra = -1;
        int64_t mine = sum_here(-1), sum;
        int64_t before = sum_before(mine, sh.scan, &sum);
        total = uniform(sum);
        if (total == 0) return false;
        if (total > groups) {
            extra = extra_;
            mine = sum_here(extra);
            __syncthreads();
            before = sum_before(mine, sh.scan, &sum);
            total = uniform(sum);
        }
        // (in cells a workgroup's range is one; a line of more than `groups` cells has more steps than workgroups)
        ng = uniform((int)min(total, (int64_t)groups));
        if ((int)blockIdx.x >= ng) return false;
        // workgroups go round-robin over the XCDs: neighbours on the line share an XCD's L2
        const int xcd = blockIdx.x % 8;
        wg = xcd * (ng / 8) + min(xcd, ng % 8) + (int)(blockIdx.x / 8);
        pos = uniform(total * wg / ng);
        hi = uniform(total * (wg + 1) / ng);
        if (pos >= before && pos < before + mine) {
            int64_t at = before;
            for (int x = 0; x < per; ++x) {
                const int64_t c = cost_of(a, x == 0 ? own : Sequence(a, tid * per + x), nhg, extra);
                if (pos < at + c) {
                    sh.found[0] = tid * per + x;
                    sh.found[1] = at;
                    break;
                }
                at += c;
            }
        }
        __syncthreads();
        b = uniform((int)sh.found[0]);
        base = uniform(sh.found[1]);
        window_at = b - 32;
        if (per == 1) {
            window_at = b;
            if (tid >= b && tid < b + 32) to_window(own, sh, tid - b);       // (past the last sequence: not looked at)
            __syncthreads();
        }
        return true;
    }

    static __device__ __forceinline__ void to_window(const Sequence& s, LineShared<THREADS>& sh, int at) {
        sh.window[0][at] = s.first;
        sh.window[1][at] = s.n;
        sh.window[2][at] = s.L;
    }

    // The next segment; false at the end of the range.  Called by all threads.
    __device__ __forceinline__ bool next(const PagedArgs& a, LineShared<THREADS>& sh) {
        while (pos < hi) {
            if (b >= window_at + 32) {
                window_at = b;
                __syncthreads();
                if (threadIdx.x < 32 && b + (int)threadIdx.x < a.B)
                    to_window(Sequence(a, b + (int)threadIdx.x), sh, (int)threadIdx.x);
                __syncthreads();
            }
            first = uniform(sh.window[0][b - window_at]);
            n = uniform(sh.window[1][b - window_at]);
            L = uniform(sh.window[2][b - window_at]);
            steps = max((L + STEP - 1) / STEP, 1);
            const int len = length(steps, extra);
            const int64_t c = units(a, n, nhg) * len;
            if (pos >= base + c) {
                base += c;
                ++b;
                continue;
            }
            const int unit = uniform((int)((pos - base) / len));
            const int tiles = (int)(((int64_t)n * (a.Hq / a.H) + ROWS - 1) / ROWS);
            hg = unit / tiles;
            rt = unit - hg * tiles;
            const int64_t at = base + (int64_t)unit * len;   // the unit's place
            if (extra < 0) {
                w0 = (int)at;
                parts = len;
                me = (int)(pos - at);
                s_in = (int)((int64_t)steps * me / len);
                count = (int)((int64_t)steps * (me + 1) / len) - s_in;
                ++pos;
                return true;
            }
            const int64_t u0 = at + extra;                   // where its steps lie
            s_in = (int)max(pos - u0, (int64_t)0);
            const int s_out = (int)min(hi - u0, (int64_t)steps);
            pos = u0 + max(s_out, 0);
            count = s_out - s_in;
            if (count <= 0) return false;                    // (its beginning alone lies at the range's end)
            w0 = workgroup_of(u0);
            parts = workgroup_of(u0 + steps - 1) - w0 + 1;
            me = wg - w0;
            return true;
        }
        return false;
    }

    __device__ __forceinline__ bool whole() const { return count == steps; }
    __device__ __forceinline__ int workgroup_of(int64_t step) const { return uniform((int)(((step + 1) * ng - 1) / total)); }
};

// The parts of a line's current unit.
template <int THREADS, int ROWS, int HG, int DP, class LINE>
struct Parts {
    static constexpr int kPart = HG * ROWS * (DP + 4);       // floats: HG heads of ROWS rows of DP sums, then each
                                                             // row's reference and sum of p, and those of a run
    float* part;
    unsigned int* tickets;
    int groups, w0, parts, me, run;

    __device__ __forceinline__ Parts(const LINE& l, float* part_, unsigned int* tickets_, int groups_)
        : part(part_), tickets(tickets_), groups(groups_), w0(l.w0), parts(l.parts), me(l.me) {
        run = parts <= 3 * kJoin / 2 ? parts : kJoin;
    }
    // (a workgroup has a part of at most one unit that starts in it, and of one that started before)
    __device__ __forceinline__ int slot(int x) const { return 2 * (w0 + x) + (x == 0 ? 1 : 0); }
    __device__ __forceinline__ float* sums(int x) const { return part + (int64_t)slot(x) * kPart; }
    __device__ __forceinline__ uint64_t* ml(int x, int round) const {
        return reinterpret_cast<uint64_t*>(sums(x) + HG * ROWS * DP) + round * HG * ROWS;
    }
    __device__ __forceinline__ void store_ml(int row, float m, float l) const {
        __hip_atomic_store(ml(me, 0) + row, two_floats(m, l), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }

    // true in the workgroup that is the last of `expected`: what the others stored is there then
    __device__ __forceinline__ bool last_of(unsigned int* ticket, int expected, LineShared<THREADS>& sh) const {
        wait_loads<0>();                                     // this wave's stores are acknowledged
        __syncthreads();
        if (threadIdx.x == 0) {
            sh.is_last = (int)__hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == expected - 1;
            if (sh.is_last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        return sh.is_last != 0;
    }

    // Parts x0, x0 + step, .. below x1, in the line's order whoever came last, to the output or to the place of
    // the first.  A thread takes four channels of K rows; Z parts of them are in flight at a time.
    __device__ __forceinline__ void join(const PagedArgs& a, const LINE& l, int x0, int x1, int step,
                                         int round, bool output) const {
        constexpr int K = 2, Z = 8;
        const int G = a.Hq / a.H, R = l.n * G;
        const int zs = (x1 - x0 + step - 1) / step, quads = a.D / 4;
        const int Rt = min(R - l.rt * ROWS, ROWS), all = min(a.H - l.hg * HG, HG) * Rt * quads;
        for (int e0 = 0; e0 < all; e0 += K * THREADS) {
            int from[K], at_row[K];
            f32x4_t acc[K];
            float mx[K], sum[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int e = min(e0 + k * THREADS + (int)threadIdx.x, all - 1), y = e / quads;
                at_row[k] = y / Rt * ROWS + y % Rt;
                from[k] = at_row[k] * DP + (e - y * quads) * 4;
                acc[k] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
                mx[k] = kLowest;
                sum[k] = 0.0f;
            }
            for (int z0 = 0; z0 < zs; z0 += Z) {
                f32x4_t v[Z][K];
                uint64_t p[Z][K];
#pragma unroll
                for (int u = 0; u < Z; ++u)
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const int x = x0 + min(z0 + u, zs - 1) * step;
                        p[u][k] = __hip_atomic_load(ml(x, round) + at_row[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        v[u][k] = load_agent(sums(x) + from[k]);
                    }
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    float top = mx[k];
#pragma unroll
                    for (int u = 0; u < Z; ++u) top = fmaxf(top, __uint_as_float((uint32_t)p[u][k]));
                    const float down = exp2_hw(mx[k] - top);
                    mx[k] = top;
                    sum[k] *= down;
                    acc[k] *= down;
#pragma unroll
                    for (int u = 0; u < Z; ++u)
                        if (z0 + u < zs) {
                            const float f = exp2_hw(__uint_as_float((uint32_t)p[u][k]) - top);
                            sum[k] += __uint_as_float((uint32_t)(p[u][k] >> 32)) * f;
                            acc[k] += v[u][k] * f;
                        }
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (e0 + k * THREADS + (int)threadIdx.x >= all) break;
                const int d = from[k] - at_row[k] * DP;
                if (output) {
                    const int h = at_row[k] / ROWS, row = l.rt * ROWS + at_row[k] % ROWS, i = row / G, g = row - i * G;
                    const bool none = sum[k] == 0.0f;
                    const float f = 1.0f / sum[k];
                    uint2 y;
                    y.x = none ? 0 : f32_to_bf16x2(acc[k][0] * f, acc[k][1] * f);
                    y.y = none ? 0 : f32_to_bf16x2(acc[k][2] * f, acc[k][3] * f);
                    *reinterpret_cast<uint2*>(a.out + (int64_t)(l.first + i) * a.ld_out +
                                              (int64_t)((l.hg * HG + h) * G + g) * a.D + d) = y;
                } else {
                    store_agent(sums(x0) + from[k], acc[k]);
                    if (d == 0)
                        __hip_atomic_store(ml(x0, 1) + at_row[k], two_floats(mx[k], sum[k]), __ATOMIC_RELAXED,
                                           __HIP_MEMORY_SCOPE_AGENT);
                }
            }
        }
    }

    // After this workgroup's part has been stored: the joins that fall to it.  Called by all threads.
    __device__ __forceinline__ void finish(const PagedArgs& a, const LINE& l, LineShared<THREADS>& sh) const {
        const int r0 = me / run * run, runs = (parts + run - 1) / run;
        if (last_of(tickets + slot(r0), min(run, parts - r0), sh)) {
            join(a, l, r0, min(r0 + run, parts), 1, 0, runs == 1);
            if (runs > 1 && last_of(tickets + 2 * groups + w0, runs, sh)) join(a, l, 0, parts, run, 1, true);
        }
        __syncthreads();
    }
};

}  // namespace

}  // namespace specfp8
