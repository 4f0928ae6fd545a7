// Attention of many rows (whole prompts, long chunks): tiles on the matrix cores.
//
// Mathematics: as in attn_stream.hpp (a running reference that moves only when
// a score exceeds it by 2^8; p rounded to bf16 for the second product; sums in
// fp32).
//
// A workgroup of 4 waves owns 128 rows -- a row is a (token, query head) pair, the
// heads of one KV head side by side, so that a causal tile's rows end within
// 128/G tokens -- and walks its keys in tiles of 64.  K and V tiles lie in LDS as
// bf16 rows, two buffers of each; every wave reads them for its own 32 rows.
//   S^T = K Q^T  on v_mfma_f32_32x32x16_bf16 (A: 32 keys x 16 channels, B: queries, held in
//     registers): a lane holds one row's scores at keys 8 (i/4) + 4 (lane/32) + i % 4.
//   O^T = V^T P^T: the probabilities of a lane are, as they are, its k-slots of the
//     second operand when V^T is read with keys in the same order; the
//     transposing LDS read (ds_read_b64_tr_b16: 4 keys of one channel per lane) does.
// Two workgroups share a CU, so that one wave's exponentials run beside the
// other's matrix instructions.
// Chunks of 16 bytes lie at slot c ^ f(key) of their row, so that the 16 lanes of
// an LDS cycle (K: lanes l and l + 16, l % 16 < 8; V: 4 keys of 64 bytes) hit different banks.
#pragma once

#include <type_traits>

#include "attn_common.hpp"

namespace specfp8 {

namespace {

template <int DP>
struct TileShape_ {
    static constexpr int kRows = 128, kKeys = 64;
    static constexpr int kRowBytes = 2 * DP;
    static constexpr int kTile = kKeys * kRowBytes;          // bytes of a K (V) tile
    static constexpr int kLds = 4 * kTile;
    static constexpr int KS = DP / 16, DB = DP / 32;         // channel steps of the scores, channel blocks of the sums
    static constexpr int kLoads = kTile / 1024 / 4;          // 1 KiB loads of a tile per wave
};

template <int DP>
__device__ __forceinline__ int tile_k_swizzle(int r) {
    if constexpr (DP == 64) return ((r >> 1) & 3) | (((r >> 4) & 1) << 2);
    else return (r & 7) | (((r >> 4) & 1) << 3);
}
template <int DP>
__device__ __forceinline__ int tile_v_swizzle(int r) {
    if constexpr (DP == 64) return ((r >> 1) & 1) << 2;
    else return (r & 3) << 2;
}

// What a wave keeps of its 32 rows.
template <int DP>
struct RowState {
    f32x16_t o[DP / 32];
    float m, l;
    uint64_t plus, minus;         // channels (16 * block + i) that +inf or NaN, and -inf or NaN, values reached
    static_assert(DP <= 128, "64 marks");
};

// Two bf16 halves that are infinite or NaN: 0x8000 in each.
__device__ __forceinline__ uint32_t not_finite(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// The keys of a tile that a row sees when these are its first `visible` ones, as a lane holds them: bit
// 32 kb + 8 (i/4) + i % 4 is key 32 kb + 8 (i/4) + 4 (lane/32) + i % 4.
__device__ __forceinline__ uint64_t seen_keys(int visible) {
    const int d = visible - 4 * (int)((threadIdx.x >> 5) & 1);
    return d <= 0 ? 0 : (d >= 64 ? ~0ull : (1ull << d) - 1);
}

// The second product's operand: 8 keys (k-slots) of one channel per lane; a lane of 16 addresses 4 channels
// of key 4 (lane/32) + its quarter.  Step u: keys 16 u .., block d: channels 32 d ..
template <int DP>
struct ValueReads {
    uint32_t va;
    __device__ __forceinline__ explicit ValueReads(uint32_t vt) {
        const int lane = threadIdx.x & 63, i16 = lane & 15, r = 4 * (lane >> 5) + (i16 >> 2);
        va = vt + r * 2 * DP + (((2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ tile_v_swizzle<DP>(r)) << 4) + 8 * (i16 & 1);
    }
    __device__ __forceinline__ u32x4_t operator()(int u, int d) const {
        typedef short i16x4_t __attribute__((ext_vector_type(4)));
        const uint32_t at = (va ^ (d << 6)) + u * 32 * DP;
        const i32x2_t a = __builtin_bit_cast(i32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((SPEC_LDS i16x4_t*)(uintptr_t)at));
        const i32x2_t b = __builtin_bit_cast(
            i32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((SPEC_LDS i16x4_t*)(uintptr_t)(at + 16 * DP)));
        return u32x4_t{(uint32_t)a[0], (uint32_t)a[1], (uint32_t)b[0], (uint32_t)b[1]};
    }
};

// One tile of 64 keys at LDS `kt`, `vt` for a wave's 32 rows.  full: every row sees all of it; otherwise a row
// sees its first `visible` keys.
template <int DP>
__device__ __forceinline__ void attend_tile(RowState<DP>& st, const bf16x8_t (&q)[DP / 16], uint32_t kt, uint32_t vt,
                                            int visible, bool full, float c2) {
    using C = TileShape_<DP>;
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31;
    // ---- scores
    const uint32_t ka = kt + l32 * C::kRowBytes + ((h ^ tile_k_swizzle<DP>(l32)) << 4);
    f32x16_t s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.0f;
    }
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const bf16x8_t kf = *(const SPEC_LDS bf16x8_t*)(uintptr_t)((ka ^ (ks << 5)) + kb * 32 * C::kRowBytes);
            s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[ks], s[kb], 0, 0, 0);
        }
    }
    if (!full) {
        const uint64_t seen = seen_keys(visible);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[kb][i] = (seen >> (32 * kb + 8 * (i / 4) + i % 4)) & 1 ? s[kb][i] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[0][i]);
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[1][i]);
    top *= c2;
    if (__ballot(top > st.m + kLazy)) {
        const float mx = fmaxf(st.m, max_halves(top));
        const float down = exp2_hw(st.m - mx);
        st.m = mx;
        st.l *= down;
#pragma unroll
        for (int d = 0; d < C::DB; ++d) st.o[d] *= down;
    }
    // ---- probabilities
    bf16x8_t p[4];
    float sum = 0.0f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 8 * (u & 1) + 2 * e;
            const float a = exp2_hw(fmaf(s[u >> 1][i], c2, -st.m)), b = exp2_hw(fmaf(s[u >> 1][i + 1], c2, -st.m));
            sum += a + b;
            w[e] = f32_to_bf16x2(a, b);
        }
        p[u] = __builtin_bit_cast(bf16x8_t, w);
    }
    st.l += sum;
    // ---- sums of values
    const ValueReads<DP> values(vt);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int d = 0; d < C::DB; ++d)
            st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, values(u, d)), p[u], st.o[d],
                                                              0, 0, 0);
}

// An infinite or NaN value reaches the rows that see its key and no others (0 * inf is NaN): in a tile that
// some row sees in part such values count 0 in the sums (clean_tile), and (keys that hold one) x (keys
// that a row sees), as products of ones, mark the channels that they reach (mark_tile).
template <int DP>
__device__ __forceinline__ void mark_tile(uint32_t vt, int visible, uint64_t& plus, uint64_t& minus) {
    using C = TileShape_<DP>;
    const uint64_t seen = seen_keys(visible);
    const ValueReads<DP> values(vt);
#pragma unroll 1
    for (int u = 0; u < 4; ++u) {
        u32x4_t sees;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            sees[e] = ones((uint32_t)(seen >> (32 * (u >> 1) + 16 * (u & 1) + 8 * (e >> 1) + 2 * (e & 1))));
#pragma unroll 1
        for (int d = 0; d < C::DB; ++d) {
            const u32x4_t v = values(u, d);
            u32x4_t up, down;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t n = not_finite(v[e]) >> 15;                                          // 1 in each half
                const uint32_t nan = (((v[e] & 0x007f007fu) + 0x007f007fu) >> 7) & 0x00010001u;
                const uint32_t neg = (v[e] >> 15) & 0x00010001u;
                const uint32_t x = n & (nan | ~neg), y = n & (nan | neg);
                up[e] = ones((x & 1u) | ((x >> 15) & 2u));
                down[e] = ones((y & 1u) | ((y >> 15) & 2u));
            }
            f32x16_t zero;
#pragma unroll
            for (int i = 0; i < 16; ++i) zero[i] = 0.0f;
            const f32x16_t hp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, up),
                                                                        __builtin_bit_cast(bf16x8_t, sees), zero, 0, 0, 0);
            const f32x16_t hm = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, down),
                                                                        __builtin_bit_cast(bf16x8_t, sees), zero, 0, 0, 0);
            uint32_t x = 0, y = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x |= (uint32_t)(hp[i] > 0.0f) << i;
                y |= (uint32_t)(hm[i] > 0.0f) << i;
            }
            plus |= (uint64_t)x << (16 * d);
            minus |= (uint64_t)y << (16 * d);
        }
    }
}

// This thread's part of the tile: whether it holds such values / without them.
template <int DP>
__device__ __forceinline__ bool wild_part(const uint8_t* tile) {
    uint32_t any = 0;
#pragma unroll
    for (int x = 0; x < TileShape_<DP>::kTile / 4096; ++x) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(tile + x * 4096 + threadIdx.x * 16);
        any |= not_finite(v[0]) | not_finite(v[1]) | not_finite(v[2]) | not_finite(v[3]);
    }
    return any != 0;
}
template <int DP>
__device__ __forceinline__ void clean_part(uint8_t* tile) {
#pragma unroll 1
    for (int x = 0; x < TileShape_<DP>::kTile / 4096; ++x) {
        u32x4_t* const at = reinterpret_cast<u32x4_t*>(tile + x * 4096 + threadIdx.x * 16);
        u32x4_t v = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] &= ~((not_finite(v[e]) >> 15) * 0xffffu);
        *at = v;
    }
}

template <int DP>
__device__ __forceinline__ void begin_rows(RowState<DP>& st) {
    st.m = kLowest;
    st.l = 0.0f;
    st.plus = st.minus = 0;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[d][i] = 0.0f;
}

// The sum of p over both halves, and the marks into the sums.
template <int DP>
__device__ __forceinline__ void end_rows(RowState<DP>& st) {
    st.l = sum_halves(st.l);
    if (__ballot((st.plus | st.minus) != 0)) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool a = (st.plus >> (16 * d + i)) & 1, b = (st.minus >> (16 * d + i)) & 1;
                if (a) st.o[d][i] += INFINITY;
                if (b) st.o[d][i] -= INFINITY;
            }
    }
}

// ---- prompts: K and V straight from bf16 rows ------------------------------------
template <int DP>
__global__ __launch_bounds__(256, 2) void prompt_tile_kernel(PromptArgs a, int slots) {
    using C = TileShape_<DP>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t tile_smem[];
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), h = lane >> 5, l32 = lane & 31;
    const int G = a.Hq / a.H;
    // The tiles of prompt b have the slots from floor(cu[b] G / 128) + b on (some stay empty): which prompt a slot
    // belongs to takes one comparison per prompt.  Late tiles, the longest, go first; heads go round-robin over the
    // XCDs, so that a KV head's tiles share an L2.
    const int head = blockIdx.x % a.H, slot = slots - 1 - (int)(blockIdx.x / a.H);
    int b = -1;
    for (int x = 0; x < a.B; x += 64) {
        const int y = x + lane;
        const bool at = y < a.B && (int64_t)min(max(a.cu[min(y, a.B)], 0), a.T) * G / C::kRows + y <= slot;
        const uint64_t votes = __ballot(at);
        if (votes) b = x + 63 - __builtin_clzll(votes);
        if (votes != ~0ull) break;
    }
    if (b < 0) return;
    int first, n;
    rows_of(a.cu, a.T, a.B, b, &first, &n);
    first = uniform(first);
    n = uniform(n);
    const int tile = slot - (int)((int64_t)first * G / C::kRows + b);
    const int64_t row0 = (int64_t)tile * C::kRows;
    if (tile < 0 || row0 >= (int64_t)n * G) return;

    // this wave's rows: queries, and the last key that each sees (its own token)
    const int64_t row = row0 + 32 * w + l32;
    const bool there = row < (int64_t)n * G;
    const int i = there ? (int)(row / G) : n - 1, g = there ? (int)(row - (int64_t)i * G) : 0;
    const uint16_t* const src = a.q + (int64_t)(first + i) * a.ld_q + (int64_t)(head * G + g) * a.D;
    bf16x8_t q[C::KS];
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
        const int d = 16 * ks + 8 * h;
        u32x4_t v = *reinterpret_cast<const u32x4_t*>(src + min(d, a.D - 8));
        if (d >= a.D) v = u32x4_t{0, 0, 0, 0};
        q[ks] = __builtin_bit_cast(bf16x8_t, v);
    }
    const int64_t last_row = min(row0 + C::kRows, (int64_t)n * G) - 1;
    const int tiles = uniform((int)(last_row / G) / C::kKeys + 1);
    const int first_token = uniform((int)(row0 / G));
    const int wave_first = uniform((int)min((row0 + 32 * w) / G, (int64_t)n - 1));          // first and last token of the wave's rows
    const int wave_last = uniform((int)(min(row0 + 32 * w + 31, last_row) / G));

    // tiles to LDS: load x of this wave covers 1024/row bytes keys from (4 x + w) ..; a lane 16 bytes of one
    const uint32_t smem = uniform((int)lds_at(tile_smem));
    constexpr int kPer = 1024 / C::kRowBytes, kChunks = DP / 8;
    const int chunks = a.D / 8, ld_key = lane / kChunks, ld_slot = lane % kChunks;
    const uint16_t* const k_rows = a.k + (int64_t)first * a.ld_k + (int64_t)head * a.D;
    const uint16_t* const v_rows = a.v + (int64_t)first * a.ld_v + (int64_t)head * a.D;
    const auto stage = [&](int t) {
        const uint32_t to = smem + (t & 1) * 2 * C::kTile;
#pragma unroll
        for (int x = 0; x < C::kLoads; ++x) {
            const int part = 4 * x + w, r = part * kPer + ld_key;
            const int64_t key = min(t * C::kKeys + r, n - 1);                   // (past the end: the last key again)
            const int ck = ld_slot ^ tile_k_swizzle<DP>(r), cv = ld_slot ^ tile_v_swizzle<DP>(r);
            load_lds16(k_rows + key * a.ld_k + (ck < chunks ? ck * 8 : 0), to + part * 1024);
            load_lds16(v_rows + key * a.ld_v + (cv < chunks ? cv * 8 : 0), to + C::kTile + part * 1024);
        }
    };
    RowState<DP> st;
    begin_rows(st);
    stage(0);
    wait_loads<0>();
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) asm volatile("" : "+v"(q[ks]));
    __syncthreads();
    const float c2 = a.scale * 1.4426950408889634f;
    for (int t = 0; t < tiles; ++t) {
        if (t + 1 < tiles) stage(t + 1);
        const uint32_t kt = smem + (t & 1) * 2 * C::kTile;
        const int k0 = t * C::kKeys;
        uint8_t* const values = tile_smem + (t & 1) * 2 * C::kTile + C::kTile;
        if (k0 + C::kKeys - 1 > first_token && __syncthreads_or(wild_part<DP>(values))) {
            mark_tile<DP>(kt + C::kTile, i + 1 - k0, st.plus, st.minus);
            __syncthreads();
            clean_part<DP>(values);
            __syncthreads();
        }
        if (k0 <= wave_last) attend_tile(st, q, kt, kt + C::kTile, i + 1 - k0, k0 + C::kKeys - 1 <= wave_first, c2);
        wait_loads<0>();
        __syncthreads();
    }
    end_rows(st);
    if (!there) return;
    const float inv = st.l == 0.0f ? 0.0f : 1.0f / st.l;
    uint16_t* const dst = a.out + (int64_t)(first + i) * a.ld_out + (int64_t)(head * G + g) * a.D + 4 * h;
#pragma unroll
    for (int d = 0; d < C::DB; ++d)
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (32 * d + 8 * x < a.D) {
                uint2 y;
                y.x = f32_to_bf16x2(st.o[d][4 * x] * inv, st.o[d][4 * x + 1] * inv);
                y.y = f32_to_bf16x2(st.o[d][4 * x + 2] * inv, st.o[d][4 * x + 3] * inv);
                *reinterpret_cast<uint2*>(dst + 32 * d + 8 * x) = y;
            }
}

}  // namespace

}  // namespace specfp8
