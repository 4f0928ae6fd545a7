// Attention of few rows over the paged FP8 cache (single tokens, drafted
// chains, trees): a stream over the cache.
//
// Mathematics.  With t_j = s_ij log2(e), a running reference m and
// p_j = 2^(t_j - m):  out = sum_j p_j v_j / sum_j p_j.  The reference moves only when a
// score exceeds it by more than 2^8 (kLazy): p then stays below 2^8, sums and
// products are fp32, and nearly every tile skips the rescale and the lane
// exchange that a maximum per tile needs.
//
// Work: attn_line.hpp; a unit is (sequence, 16*NQ rows, HG KV heads).
// A wave owns one KV head and every KW-th tile of 32 keys, for all rows of the unit:
// no data is shared between waves, so nothing waits at a barrier until the
// end of a unit.  Codes go from HBM to LDS without registers (16 bytes per
// lane from its key's page) into a ring of two stages; table entries of the tile
// after next travel the same way.
//   S^T = K Q^T  on v_mfma_f32_16x16x32_bf16: codes are exact in bf16.  A lane holds
//     the scores of one row (lane % 16) at keys 4 (lane/16) + 0..3 and 16 more.
//   O^T = V^T P^T: the 8 probabilities of a lane are, as they are, the 8 k-slots of
//     its operand when V^T is read with keys in the same order, which the
//     transposing LDS read (ds_read_b64_tr_b8, 8 keys of one channel per lane) does.
// Chunks of a row lie at slot c ^ f(key) so that the 16 lanes that an LDS cycle
// serves hit different banks.
//
// What bounds it: the cache's bytes.  At 8 KV heads of 128, 4 query heads each: two contexts of 95000 tokens
// and one row each take 86 us (404 MB, 4.7 TB/s with the start and the join; 5.8 to 6.2 inside the loop), 64
// of 512..4096 tokens 68 us with one row each and 90 with five: there a range holds 1.5 and 2 parts of units on
// average, and each begins with loads that depend on each other (tables, offsets, the first codes) and ends in a
// join.  Not faster: rings of 3 and 4 stages, eight waves a workgroup, a raised wave priority.
#pragma once

#include <type_traits>

#include "attn_line.hpp"

namespace specfp8 {

namespace {


// LDS slot of 16-byte chunk c of key row r (0..31): c ^ this.  K: lanes l and l+16 (l % 16 < 8) are
// served together, rows 0..7 at chunks 2x and 2x+1.  V: lanes 0..31, 16 rows (0..7
// and 16..23, or 8..15 and 24..31) at one chunk.  Rows of DP bytes: 256/DP of
// them share one line of banks.
template <int DP>
__device__ __forceinline__ int k_swizzle(int r) {
    if constexpr (DP == 64) return 2 * ((r >> 2) & 1);
    else if constexpr (DP == 128) return 2 * ((r >> 1) & 3);
    else return 2 * (r & 7);
}
template <int DP>
__device__ __forceinline__ int v_swizzle(int r) {
    if constexpr (DP == 64) return ((r >> 2) & 1) | (((r >> 4) & 1) << 1);
    else if constexpr (DP == 128) return ((r >> 1) & 3) | (((r >> 4) & 1) << 2);
    else return (r & 7) | (((r >> 4) & 1) << 3);
}

constexpr int kStreamCell = 3;                               // steps that are worth a join (1, 2, 4: slower on short lines)

constexpr int kStreamWaves = 4;                              // of a workgroup

template <int DP, int NQ, int HG>
struct StreamShape {
    static constexpr int KW = kStreamWaves / HG;             // waves that share a head
    static constexpr int kRows = 16 * NQ;
    static constexpr int kStep = 32 * KW;                    // keys of a step
    static constexpr int kTile = 32 * DP;                    // bytes of a tile's K (V) codes
    static constexpr int kStage = 2 * kTile + 256;           // and 64 scales
    static constexpr int kTables = 2 * kStage;               // two tiles' table entries
    static constexpr int kOffs = kTables + 2 * 256;          // byte offsets of a tile's rows
    static constexpr int kWave = (kOffs + 256 + DP - 1) / DP * DP;
    static constexpr int kLds = kStreamWaves * kWave;
    static constexpr int kBlocks = DP / 16;
    static_assert(kStage % DP == 0 && kWave % DP == 0, "a V row's address has no bits where its chunks' are");
    static_assert(KW == 1 || kStreamWaves / 2 * NQ * (kBlocks * 256 + 128) * 4 <= kLds, "half the waves' results fit for the join");
};

template <int DP, int NQ, int HG>
__global__ __launch_bounds__(64 * kStreamWaves, DP == 256 ? 1 : 2) void paged_stream_kernel(PagedArgs a, float* part,
                                                                                 unsigned int* tickets, int groups, int extra) {
    using C = StreamShape<DP, NQ, HG>;
    constexpr int kThreads = 64 * kStreamWaves;
    constexpr int NB = C::kBlocks, KS = DP / 64;
    // (sized at the launch: with the size in its view the compiler counts on one workgroup per CU, and then keeps the
    // sums in AGPRs and copies them for every rescale)
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    __shared__ LineShared<kThreads> sh;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.Hq / a.H;
    const int q16 = lane & 15, qd = lane >> 4;

    Line<kThreads, C::kRows, C::kStep, kStreamCell> line;
    if (!line.begin(a, sh, HG, groups, extra)) return;

    // ---- this wave's corner of LDS
    const int hw = w % HG, kw = w / HG;
    uint8_t* const ring = smem + w * C::kWave;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_at(ring));
    const uint32_t* const tab = reinterpret_cast<const uint32_t*>(ring + C::kTables);
    int64_t* const offs = reinterpret_cast<int64_t*>(ring + C::kOffs);
    // loads of K and V: lane -> key row and chunk of the 1 KiB of a load
    constexpr int kKeys = 1024 / DP;                         // keys of a load
    const int ld_key = lane / (DP / 16), ld_slot = lane % (DP / 16);
    const int chunks = a.D / 16;
    const int bs = a.block_size, step_q = C::kStep / bs, step_r = C::kStep % bs;
    const int last_block = max(a.max_len / bs - 1, 0);
    // (as a scalar of its own: a loop that reads one field of the arguments keeps, or reloads, eight)
    const uint32_t num_blocks = uniform(a.num_blocks), head_size = uniform(a.D);
    const int heads = uniform(a.H), per_tensor = uniform(a.per_tensor);
    const float* const scales = lane < 32 ? a.k_scale : a.v_scale;
    const uint32_t page_rows = bs * a.H, page_bytes = page_rows * a.D;          // (a page has less than 4 GiB of codes)
    const float c2 = a.scale * 1.4426950408889634f;

    while (line.next(a, sh)) {
        const int first = line.first, n = line.n, L = line.L, rt = line.rt, hg = line.hg, s_in = line.s_in, count = line.count;
        const int b = line.b;
        const int R = n * G, head = hg * HG + hw;
        const bool active = head < a.H;

        f32x4_t o[NQ][NB];
        float m[NQ], l[NQ];
#pragma unroll
        for (int x = 0; x < NQ; ++x) {
            m[x] = kLowest;
            l[x] = 0.0f;
#pragma unroll
            for (int d = 0; d < NB; ++d) o[x][d] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
        if (active) {
            // ---- the rows: queries, and what each sees
            bf16x8_t q[NQ][KS][2];
            int lim[NQ];
            std::conditional_t<(NB > 8), uint64_t, uint32_t> marked[NQ];          // channels of this lane that a NaN code reached
            uint64_t tree[NQ];
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                const int row = rt * C::kRows + x * 16 + q16, i = row / G, g = row - i * G;
                const bool there = row < R;
                const uint16_t* src = a.q + (int64_t)(first + (there ? i : 0)) * a.ld_q + (int64_t)(head * G + (there ? g : 0)) * a.D;
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int d = 64 * s + 16 * qd + 8 * u;
                        // (a row that is not there reads the first; a channel past the head's end becomes 0)
                        u32x4_t v = *reinterpret_cast<const u32x4_t*>(src + min(d, a.D - 8));
                        if (d >= a.D) v = u32x4_t{0, 0, 0, 0};
                        q[x][s][u] = __builtin_bit_cast(bf16x8_t, v);
                    }
                marked[x] = 0;
                lim[x] = there ? L - n + i : -1;
                tree[x] = a.tree && there && i > 0 ? a.tree[(int64_t)b * a.N + i - 1] : 0;
                if (a.tree) lim[x] = there ? L - 1 : -1;
            }
            const int all_see = a.tree ? L - a.N - 1 : L - n + rt * C::kRows / G;   // tokens up to here are seen by every row

            // ---- the ring
            const int32_t* const table = a.max_len > 0 ? a.tables + (int64_t)b * a.ld_tables : a.kv_lens;
            const int key = lane & 31;
            const int first_key = 32 * (s_in * C::KW + kw);
            int blk = (first_key + key) / bs, off_t = (first_key + key) - blk * bs, off_p = off_t;
            const auto load_table = [&](int t) {
                load_lds4(table + min(blk, last_block), ring_at + C::kTables + (t & 1) * 256);
                off_t += step_r;
                blk += step_q;
                if (off_t >= bs) {
                    off_t -= bs;
                    ++blk;
                }
            };
            int next_key = first_key;
            const auto prepare = [&](int t) -> uint32_t {            // byte offsets and scales of tile t; which keys there are
                const int page = (int)tab[(t & 1) * 64 + lane];
                const bool there = (next_key + key < L) & ((uint32_t)page < num_blocks);
                const uint32_t pg = there ? page : 0, in = (there ? off_p : 0) * heads + head;
                const uint64_t row = (uint64_t)pg * page_rows + in;
                if (lane < 32) offs[key] = (int64_t)((uint64_t)pg * page_bytes + in * head_size);
                load_lds4(scales + (per_tensor ? 0 : row), ring_at + (t & 1) * C::kStage + 2 * C::kTile);
                off_p += step_r;
                if (off_p >= bs) off_p -= bs;
                next_key += C::kStep;
                return (uint32_t)__ballot(there);
            };
            const auto load_codes = [&](int t) {
                const uint32_t to = ring_at + (t & 1) * C::kStage;
#pragma unroll
                for (int x = 0; x < C::kTile / 1024; ++x) {
                    const int r = x * kKeys + ld_key;
                    const int64_t at_row = offs[r];
                    const int ck = ld_slot ^ k_swizzle<DP>(r), cv = ld_slot ^ v_swizzle<DP>(r);
                    // (chunks past the head's end: the row's first one; their queries are 0)
                    load_lds16(a.k_cache + at_row + (ck < chunks ? ck * 16 : 0), to + x * 1024);
                    load_lds16(a.v_cache + at_row + (cv < chunks ? cv * 16 : 0), to + C::kTile + x * 1024);
                }
            };
            // A tile's group of loads: its scales, the table entries that the next group needs, its codes.
            const auto load_group = [&](int t) -> uint32_t {
                const uint32_t there = prepare(t);
                if (t + 1 < count) load_table(t + 1);
                load_codes(t);
                return there;
            };
            wait_lds();
            load_table(0);
            wait_loads<0>();
            // (the queries, too: a wait for them in the loop would drain the ring)
#pragma unroll
            for (int x = 0; x < NQ; ++x)
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(q[x][s][u]));
            uint32_t there = load_group(0);

            // One tile; full: every row sees every key of it.
            const auto attend = [&](int t, int k0, uint32_t there, bool full) {
                const uint32_t stage = ring_at + (t & 1) * C::kStage;
                const uint8_t* const kt = ring + (t & 1) * C::kStage;
                const float* const sc = reinterpret_cast<const float*>(kt + 2 * C::kTile);

                // ---- scores
                f32x4_t s[2][NQ];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                    for (int x = 0; x < NQ; ++x) s[kb][x] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int u = 0; u < KS; ++u) {
                        const int r = kb * 16 + q16;
                        const u32x4_t c = *reinterpret_cast<const u32x4_t*>(
                            kt + r * DP + (((4 * u + qd) ^ k_swizzle<DP>(r)) << 4));
                        const bf16x8_t lo8 = codes_to_bf16(c[0], c[1]), hi8 = codes_to_bf16(c[2], c[3]);
#pragma unroll
                        for (int x = 0; x < NQ; ++x) {
                            s[kb][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo8, q[x][u][0], s[kb][x], 0, 0, 0);
                            s[kb][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi8, q[x][u][1], s[kb][x], 0, 0, 0);
                        }
                    }
                }
                // values, read ahead of their use: lane j of 16 addresses half j % 2 of key row 16 (j/8) + 4 qd + (j/2) % 4
                const int vr = 16 * (q16 >> 3) + 4 * qd + ((q16 >> 1) & 3);
                const uint32_t vat = stage + C::kTile + vr * DP + (v_swizzle<DP>(vr) << 4) + 8 * (q16 & 1);
                const auto values_at = [&](int d) {
                    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((SPEC_LDS i32x2_t*)(uintptr_t)(vat ^ (d << 4)));
                };
                i32x2_t vc[NB];
#pragma unroll
                for (int d = 0; d < NB; ++d) vc[d] = values_at(d);
                const f32x4_t sk0 = *reinterpret_cast<const f32x4_t*>(sc + 4 * qd) * c2;
                const f32x4_t sk1 = *reinterpret_cast<const f32x4_t*>(sc + 16 + 4 * qd) * c2;
                const f32x4_t sv0 = *reinterpret_cast<const f32x4_t*>(sc + 32 + 4 * qd);
                const f32x4_t sv1 = *reinterpret_cast<const f32x4_t*>(sc + 48 + 4 * qd);
                // p < 2^8: its product with a value scale below 2^119 is finite, and so is what the upper half leaves.  (The
                // check takes 0.5% of a call, 2 to 3% at heads of 64; one scale a lane, or only where the reference moves:
                // no less.)
                float sv_top = fmaxf(fabsf(sv0[0]), fabsf(sv1[0]));
#pragma unroll
                for (int r = 1; r < 4; ++r) sv_top = fmaxf(sv_top, fmaxf(fabsf(sv0[r]), fabsf(sv1[r])));
                const bool huge = __ballot(sv_top >= 0x1p119f) != 0;
                uint32_t seen[NQ];
                float top[NQ];
                bool over = false;
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s[0][x][r] *= sk0[r];
                        s[1][x][r] *= sk1[r];
                    }
                    if (!full) {
                        uint32_t see = 0;
                        const int d = lim[x] - k0;
                        if (d >= 0) see = d >= 31 ? 0xffffffffu : (2u << d) - 1u;
                        if (a.tree) {
                            const int f = k0 - (L - a.N);                         // node number of the tile's first key
                            if (f >= 0) see &= f < 64 ? (uint32_t)(tree[x] >> f) : 0u;
                            else if (f > -32) see &= (uint32_t)(tree[x] << -f) | ((1u << -f) - 1u);
                        }
                        see &= there;
                        seen[x] = see >> (4 * qd);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            s[0][x][r] = (seen[x] >> r) & 1 ? s[0][x][r] : -INFINITY;
                            s[1][x][r] = (seen[x] >> (16 + r)) & 1 ? s[1][x][r] : -INFINITY;
                        }
                    }
                    float t0 = fmaxf(fmaxf(s[0][x][0], s[0][x][1]), fmaxf(s[0][x][2], s[0][x][3]));
                    float t1 = fmaxf(fmaxf(s[1][x][0], s[1][x][1]), fmaxf(s[1][x][2], s[1][x][3]));
                    top[x] = fmaxf(t0, t1);
                    over = over || top[x] > m[x] + kLazy;
                }
                if (__ballot(over)) {
#pragma unroll
                    for (int x = 0; x < NQ; ++x) {
                        const float mx = fmaxf(m[x], max_quarters(top[x]));
                        const float down = exp2_hw(m[x] - mx);
                        m[x] = mx;
                        l[x] *= down;
#pragma unroll
                        for (int d = 0; d < NB; ++d) o[x][d] *= down;
                    }
                }
                // ---- probabilities, as the second product's operand
                // (in two halves, the upper 8 bits of each and bf16 of the rest: one half alone adds as much error to a
                // row as the output's own rounding, and for few keys the same one to all its channels)
                bf16x8_t pv[NQ], rest[NQ];
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
                    float p0[4], p1[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        p0[r] = exp2_hw(s[0][x][r] - m[x]);
                        p1[r] = exp2_hw(s[1][x][r] - m[x]);
                    }
                    l[x] += ((p0[0] + p0[1]) + (p0[2] + p0[3])) + ((p1[0] + p1[1]) + (p1[2] + p1[3]));
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        p0[r] *= sv0[r];
                        p1[r] *= sv1[r];
                        if (!full) {                     // an infinite or NaN scale of a key not seen
                            p0[r] = (seen[x] >> r) & 1 ? p0[r] : 0.0f;
                            p1[r] = (seen[x] >> (16 + r)) & 1 ? p1[r] : 0.0f;
                        }
                    }
                    u32x4_t v, y;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float lo = r < 2 ? p0[2 * r] : p1[2 * r - 4], hi = r < 2 ? p0[2 * r + 1] : p1[2 * r - 3];
                        const uint32_t lo_up = __float_as_uint(lo) & 0xffff0000u, hi_up = __float_as_uint(hi) & 0xffff0000u;
                        v[r] = hi_up | (lo_up >> 16);
                        y[r] = f32_to_bf16x2(lo - __uint_as_float(lo_up), hi - __uint_as_float(hi_up));
                    }
                    if (huge) {                          // an infinite product is its upper half alone (inf - inf is NaN)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if ((v[r] & 0x7f80u) == 0x7f80u) y[r] &= 0xffff0000u;
                            if ((v[r] & 0x7f800000u) == 0x7f800000u) y[r] &= 0xffffu;
                        }
                    }
                    pv[x] = __builtin_bit_cast(bf16x8_t, v);
                    rest[x] = __builtin_bit_cast(bf16x8_t, y);
                }
                // ---- sums of values
                if (!full) {
                    // Keys that are not there: code 0.  A NaN code reaches the rows that see its key and no others
                    // (0 * NaN is NaN): it counts 0 in the sums, and its rows are marked.
                    const uint32_t keep0 = ((((there >> (4 * qd)) & 15u) * 0x00204081u) & 0x01010101u) * 0xffu;
                    const uint32_t keep1 = ((((there >> (16 + 4 * qd)) & 15u) * 0x00204081u) & 0x01010101u) * 0xffu;
                    uint32_t nans = 0;
#pragma unroll
                    for (int d = 0; d < NB; ++d) {
                        const uint32_t c0 = (uint32_t)vc[d][0] & keep0, c1 = (uint32_t)vc[d][1] & keep1;
                        const uint32_t n0 = nan_bytes(c0) >> 7, n1 = nan_bytes(c1) >> 7;
                        nans |= n0 | n1;
                        vc[d][0] = (int)(c0 & ~(n0 * 0xffu));
                        vc[d][1] = (int)(c1 & ~(n1 * 0xffu));
                    }
                    if (__ballot(nans != 0)) {
                        // (keys that hold one) x (keys that a row sees), as a product of ones
#pragma unroll 1
                        for (int d = 0; d < NB; ++d) {
                            const i32x2_t c = values_at(d);
                            const uint32_t n0 = nan_bytes((uint32_t)c[0] & keep0) >> 7;
                            const uint32_t n1 = nan_bytes((uint32_t)c[1] & keep1) >> 7;
                            u32x4_t has;
                            has[0] = ones((n0 & 1u) | ((n0 >> 7) & 2u));
                            has[1] = ones(((n0 >> 16) & 1u) | ((n0 >> 23) & 2u));
                            has[2] = ones((n1 & 1u) | ((n1 >> 7) & 2u));
                            has[3] = ones(((n1 >> 16) & 1u) | ((n1 >> 23) & 2u));
#pragma unroll
                            for (int x = 0; x < NQ; ++x) {
                                u32x4_t sees;
#pragma unroll
                                for (int y = 0; y < 4; ++y) sees[y] = ones(seen[x] >> ((y >> 1) * 16 + (y & 1) * 2));
                                const f32x4_t hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                    __builtin_bit_cast(bf16x8_t, has), __builtin_bit_cast(bf16x8_t, sees),
                                    f32x4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
                                for (int r = 0; r < 4; ++r)
                                    marked[x] |= (decltype(marked[x] + 0))(hits[r] > 0.0f ? 1 : 0) << (4 * d + r);
                            }
                        }
                    }
                }
#pragma unroll
                for (int d = 0; d < NB; ++d) {
                    const bf16x8_t vt = codes_to_bf16((uint32_t)vc[d][0], (uint32_t)vc[d][1]);
#pragma unroll
                    for (int x = 0; x < NQ; ++x) {
                        o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pv[x], o[x][d], 0, 0, 0);
                        o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, rest[x], o[x][d], 0, 0, 0);
                    }
                }
            };

            for (int t = 0; t < count; ++t) {
                wait_loads<0>();                         // the codes of t; those of t + 1 travel under its products
                wait_lds();
                uint32_t next = 0;
                if (t + 1 < count) next = load_group(t + 1);
                const int k0 = first_key + t * C::kStep;
                attend(t, k0, there, there == 0xffffffffu && k0 + 31 <= all_see);
                there = next;
            }
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                l[x] = sum_quarters(l[x]);
                if (__ballot(marked[x] != 0)) {
#pragma unroll
                    for (int d = 0; d < NB; ++d)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if ((marked[x] >> (4 * d + r)) & 1) o[x][d][r] = __builtin_nanf("");
                }
            }
        }

        // ---- waves that share a head join through LDS (odd ones into even ones, then 2 into 0)
        if constexpr (C::KW > 1) {
            float* const box = reinterpret_cast<float*>(smem);
#pragma unroll
            for (int gap = 1; gap < C::KW; gap *= 2) {
                __syncthreads();
                const bool gives = (kw & (2 * gap - 1)) == gap, takes = (kw & (2 * gap - 1)) == 0;
                float* const to = box + ((kw / (2 * gap)) * HG + hw) * (NQ * (NB * 256 + 128));
                if (gives) {
#pragma unroll
                    for (int x = 0; x < NQ; ++x) {
#pragma unroll
                        for (int d = 0; d < NB; ++d)
                            *reinterpret_cast<f32x4_t*>(to + x * (NB * 256 + 128) + d * 256 + lane * 4) = o[x][d];
                        to[x * (NB * 256 + 128) + NB * 256 + lane] = m[x];
                        to[x * (NB * 256 + 128) + NB * 256 + 64 + lane] = l[x];
                    }
                }
                __syncthreads();
                if (takes) {
#pragma unroll
                    for (int x = 0; x < NQ; ++x) {
                        const float mo = to[x * (NB * 256 + 128) + NB * 256 + lane];
                        const float lo2 = to[x * (NB * 256 + 128) + NB * 256 + 64 + lane];
                        const float mx = fmaxf(m[x], mo), da = exp2_hw(m[x] - mx), db = exp2_hw(mo - mx);
                        m[x] = mx;
                        l[x] = l[x] * da + lo2 * db;
#pragma unroll
                        for (int d = 0; d < NB; ++d) {
                            const f32x4_t v =
                                *reinterpret_cast<const f32x4_t*>(to + x * (NB * 256 + 128) + d * 256 + lane * 4);
                            o[x][d] = o[x][d] * da + v * db;
                        }
                    }
                }
            }
            __syncthreads();
        }

        const auto store_rows = [&](int x, int h, float total_l, const f32x4_t (&v)[NB]) {
            const int row = rt * C::kRows + x * 16 + q16, i = row / G, g = row - i * G;
            if (row >= R) return;
            const bool none = total_l == 0.0f;               // (zeros, whatever the values that had no weight)
            const float inv = 1.0f / total_l;
            uint16_t* const dst = a.out + (int64_t)(first + i) * a.ld_out + (int64_t)(h * G + g) * a.D + 4 * qd;
#pragma unroll
            for (int d = 0; d < NB; ++d) {
                if (16 * d < a.D) {
                    uint2 y;
                    y.x = none ? 0 : f32_to_bf16x2(v[d][0] * inv, v[d][1] * inv);
                    y.y = none ? 0 : f32_to_bf16x2(v[d][2] * inv, v[d][3] * inv);
                    *reinterpret_cast<uint2*>(dst + 16 * d) = y;
                }
            }
        };

        if (line.whole()) {
            if (active && kw == 0) {
#pragma unroll
                for (int x = 0; x < NQ; ++x) store_rows(x, head, l[x], o[x]);
            }
        } else {
            const Parts<kThreads, C::kRows, HG, DP, decltype(line)> parts(line, part, tickets, groups);
            if (active && kw == 0) {
                float* const to = parts.sums(parts.me) + hw * C::kRows * DP;
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
                    if (rt * C::kRows + x * 16 + q16 < R) {
#pragma unroll
                        for (int d = 0; d < NB; ++d)
                            if (16 * d < a.D) store_agent(to + (x * 16 + q16) * DP + 16 * d + 4 * qd, o[x][d]);
                        if (qd == 0) parts.store_ml(hw * C::kRows + x * 16 + q16, m[x], l[x]);
                    }
                }
            }
            parts.finish(a, line, sh);
        }
    }
}

}  // namespace

}  // namespace specfp8
