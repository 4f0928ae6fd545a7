// Attention of many rows (whole prompts, long chunks): tiles on the matrix cores.
//
// Mathematics: as in attn_stream.hpp (a running reference that moves only when
// a score exceeds it by 2^8; p rounded to bf16 for the second product, to two in rows of few keys; sums in
// fp32).
//
// A wave owns 32 rows, a workgroup 128 (4 waves), over the cache at heads of 128 256 (8 waves) -- a row is a
// (token, query head) pair, the heads of one KV head side by side, so that a causal tile's rows end within
// 128/G tokens -- and walks its keys in tiles of 64.  K and V tiles lie in LDS as
// bf16 rows, two buffers of each; every wave reads them for its own 32 rows.
//   S^T = K Q^T  on v_mfma_f32_32x32x16_bf16 (A: 32 keys x 16 channels, B: queries, held in
//     registers): a lane holds one row's scores at keys 8 (i/4) + 4 (lane/32) + i % 4.
//   O^T = V^T P^T: the probabilities of a lane are, as they are, its k-slots of the
//     second operand when V^T is read with keys in the same order; the
//     transposing LDS read (ds_read_b64_tr_b16: 4 keys of one channel per lane) does.
// Two waves share a SIMD, so that one's exponentials run beside the other's matrix instructions: of two workgroups
// (heads of 64, prompts of 128) or of one of eight waves (128 KB of LDS: the cache at heads of 128).  Heads of 256 take
// all registers: one wave a SIMD.
// Chunks of 16 bytes lie at slot c ^ f(key) of their row, so that the 16 lanes of
// an LDS cycle (K: lanes l and l + 16, l % 16 < 8; V: 4 keys of 64 bytes) hit different banks.
//
// What bounds it: the matrix cores and the vector instructions beside them.  A prompt of 8191 tokens, 32 query and 8 KV
// heads of 128, takes 520 to 548 us, 1.0 PFLOP/s (a large bf16 product of the card's library: 1.22), with the matrix
// cores at work 49% of the time and the vector units 45%; 9 prompts of 200..2100 tokens 156 us: each 128 rows begin with
// an empty pipeline and end in a tile that is seen in part.  Over the cache the same tile also turns 64 keys' codes into
// bf16 and scales scores and probabilities per key: 6 chunks of up to 2000 rows over 100..6000 tokens take 720 us, 0.66
// PFLOP/s (26% and 39%); 256 rows a workgroup share that work (128: a sixth more).  Not faster: the scores of the next
// tile under the sums of this one (spills), a raised wave priority, output rows through LDS.
#pragma once

#include <type_traits>

#include "attn_line.hpp"

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

// Rows of tiles whose first row sees at most this many keys keep their weights to 16 bits, as few rows do: a weight's
// rounding is most of the error of a row of few keys, and the same one in all its channels.  One tile of keys: prompts
// of 1..130 tokens take 9.0 us as before (128: 10.8), one of 8191 538 (531).  For every row: 848 us, nine prompts 236 (158).
constexpr int kFewKeys = 64;
// What a wave keeps of its 32 rows.
template <int DP>
struct RowState {
    f32x16_t o[DP / 32];
    float m, l;
    uint64_t plus[(DP + 127) / 128], minus[(DP + 127) / 128];     // channels (16 * block + i) that +inf or NaN, and
                                                                  // -inf or NaN, values reached
};

// Two bf16 halves that are infinite or NaN: 0x8000 in each.
__device__ __forceinline__ uint32_t not_finite(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }

// The first `visible` keys of a tile, as bits.
__device__ __forceinline__ uint64_t first_keys(int visible) {
    return visible <= 0 ? 0 : (visible >= 64 ? ~0ull : (1ull << visible) - 1);
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
// sees the keys of `row_sees`.  SCALED: keys and values have scales of their own in LDS, the keys' with c2 in them.
// odd: c2 is no positive finite number (a tensor's scale of 0, say), and scores take it before unseen ones become -inf.
// both: weights enter the second product as two bf16, each rounded and what that leaves (in a pass of its own: in the
// first one, before its products, it takes the registers of the tiles that do without).
template <int DP, bool SCALED>
__device__ __forceinline__ void attend_tile(RowState<DP>& st, const bf16x8_t (&q)[DP / 16], uint32_t kt, uint32_t vt,
                                            uint64_t row_sees, bool full, float c2, bool odd, bool both,
                                            const float* k_scales, const float* v_scales) {
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
    const bool fresh = st.m == kLowest;                      // (no reference yet)
    if constexpr (SCALED) {
        const float ref = fresh ? 0.0f : st.m;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const f32x4_t f = *reinterpret_cast<const f32x4_t*>(k_scales + 8 * x + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e)                      // over the reference already: one instruction, not two
                s[x >> 2][4 * (x & 3) + e] = fmaf(s[x >> 2][4 * (x & 3) + e], f[e], -ref);
        }
    }
    if (!SCALED && odd) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][i] *= c2;
        c2 = 1.0f;
    }
    if (!full) {
        const uint64_t seen = row_sees >> (4 * h);           // bit 32 kb + 8 (i/4) + i % 4: key 4 h further
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
    if constexpr (!SCALED) top *= c2;
    if (SCALED ? __ballot(top > kLazy || (fresh && top > kLowest)) : __ballot(top > st.m + kLazy)) {
        float down;
        if constexpr (SCALED) {
            const float mx = max_halves(top);
            const float up = fresh ? (mx > kLowest ? mx : 0.0f) : fmaxf(0.0f, mx);
            down = fresh ? 1.0f : exp2_hw(-up);
            st.m = fresh ? (mx > kLowest ? mx : kLowest) : st.m + up;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][i] -= up;
        } else {
            const float mx = fmaxf(st.m, max_halves(top));
            down = exp2_hw(st.m - mx);
            st.m = mx;
        }
        st.l *= down;
#pragma unroll
        for (int d = 0; d < C::DB; ++d) st.o[d] *= down;
    }
    // ---- probabilities: two at a time, those of element i of step u
    float sum = 0.0f;
    const auto weights = [&](int u, int e) -> float2 {
        const int i = 8 * (u & 1) + 2 * e;
        float a, b;
        if constexpr (SCALED) {
            a = exp2_hw(s[u >> 1][i]);
            b = exp2_hw(s[u >> 1][i + 1]);
        } else {
            a = exp2_hw(fmaf(s[u >> 1][i], c2, -st.m));
            b = exp2_hw(fmaf(s[u >> 1][i + 1], c2, -st.m));
        }
        sum += a + b;
        if constexpr (SCALED) {
            const float2 f = *reinterpret_cast<const float2*>(v_scales + 16 * u + 8 * (e >> 1) + 4 * h + 2 * (e & 1));
            a *= f.x;
            b *= f.y;
        }
        return float2{a, b};
    };
    bf16x8_t p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        u32x4_t w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 x = weights(u, e);
            w[e] = f32_to_bf16x2(x.x, x.y);
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
    if (__builtin_expect(both, false)) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            u32x4_t w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 x = weights(u, e);
                const uint32_t up = f32_to_bf16x2(x.x, x.y);
                // (an infinite weight is its upper half alone: inf - inf is NaN)
                w[e] = f32_to_bf16x2(fabsf(x.x) < INFINITY ? x.x - __uint_as_float(up << 16) : 0.0f,
                                     fabsf(x.y) < INFINITY ? x.y - __uint_as_float(up & 0xffff0000u) : 0.0f);
            }
#pragma unroll
            for (int d = 0; d < C::DB; ++d)
                st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, values(u, d)),
                                                                  __builtin_bit_cast(bf16x8_t, w), st.o[d], 0, 0, 0);
        }
    }
}

// An infinite or NaN value reaches the rows that see its key and no others (0 * inf is NaN): in a tile that
// some row sees in part such values count 0 in the sums (clean_tile), and (keys that hold one) x (keys
// that a row sees), as products of ones, mark the channels that they reach (mark_tile).
template <int DP>
__device__ __forceinline__ void mark_tile(RowState<DP>& st, uint32_t vt, uint64_t row_sees) {
    using C = TileShape_<DP>;
    const uint64_t seen = row_sees >> (4 * ((threadIdx.x >> 5) & 1));
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
#pragma unroll
            for (int z = 0; z < (DP + 127) / 128; ++z) {
                st.plus[z] |= d >> 2 == z ? (uint64_t)x << (16 * (d & 3)) : 0;
                st.minus[z] |= d >> 2 == z ? (uint64_t)y << (16 * (d & 3)) : 0;
            }
        }
    }
}

// This thread's part of the tile: whether it holds such values / without them.  16 bytes of key
// (threadIdx.x + 256 x) / (DP / 8) at a time.
template <int DP>
__device__ __forceinline__ bool wild_part(const uint8_t* tile) {
    uint32_t any = 0;
    for (int x = threadIdx.x * 16; x < TileShape_<DP>::kTile; x += blockDim.x * 16) {
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(tile + x);
        any |= not_finite(v[0]) | not_finite(v[1]) | not_finite(v[2]) | not_finite(v[3]);
    }
    return any != 0;
}
template <int DP>
__device__ __forceinline__ void clean_part(uint8_t* tile) {
#pragma unroll 1
    for (int x = threadIdx.x * 16; x < TileShape_<DP>::kTile; x += blockDim.x * 16) {
        u32x4_t* const at = reinterpret_cast<u32x4_t*>(tile + x);
        u32x4_t v = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] &= ~((not_finite(v[e]) >> 15) * 0xffffu);
        *at = v;
    }
}

// Keys that are not there have values 0; keys whose value scale is infinite or NaN have their values scaled by it
// here (infinite or NaN, so that they are marked) and no weight.
template <int DP>
__device__ __forceinline__ void settle_part(uint8_t* tile, uint64_t there, const float* v_scales) {
#pragma unroll 1
    for (int x = threadIdx.x * 16; x < TileShape_<DP>::kTile; x += blockDim.x * 16) {
        const int key = x / (2 * DP);
        u32x4_t* const at = reinterpret_cast<u32x4_t*>(tile + x);
        if (!((there >> key) & 1)) {
            *at = u32x4_t{0, 0, 0, 0};
        } else if (v_scales && !(fabsf(v_scales[key]) < INFINITY)) {
            const float f = v_scales[key];
            u32x4_t v = *at;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = f32_to_bf16x2(__uint_as_float(v[e] << 16) * f, __uint_as_float(v[e] & 0xffff0000u) * f);
            *at = v;
        }
    }
}

template <int DP>
__device__ __forceinline__ void begin_rows(RowState<DP>& st) {
    st.m = kLowest;
    st.l = 0.0f;
#pragma unroll
    for (int z = 0; z < (DP + 127) / 128; ++z) st.plus[z] = st.minus[z] = 0;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) st.o[d][i] = 0.0f;
}

// The sum of p over both halves, and the marks into the sums.
template <int DP>
__device__ __forceinline__ void end_rows(RowState<DP>& st) {
    st.l = sum_halves(st.l);
    uint64_t any = 0;
#pragma unroll
    for (int z = 0; z < (DP + 127) / 128; ++z) any |= st.plus[z] | st.minus[z];
    if (__ballot(any != 0)) {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int at = 16 * (d & 3) + i;
                if ((st.plus[d >> 2] >> at) & 1) st.o[d][i] += INFINITY;
                if ((st.minus[d >> 2] >> at) & 1) st.o[d][i] -= INFINITY;
            }
    }
}

// The rows' results as bf16: channels 32 d + 8 x + 4 (lane/32) .. of this lane's row, `dst` its first channel.
template <int DP>
__device__ __forceinline__ void store_rows(const RowState<DP>& st, uint16_t* dst, int D, float scale) {
    const bool none = st.l == 0.0f;                          // (zeros, whatever the values that had no weight)
    const float inv = scale / st.l;
    dst += 4 * ((threadIdx.x >> 5) & 1);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (32 * d + 8 * x < D) {
                uint2 y;
                y.x = none ? 0 : f32_to_bf16x2(st.o[d][4 * x] * inv, st.o[d][4 * x + 1] * inv);
                y.y = none ? 0 : f32_to_bf16x2(st.o[d][4 * x + 2] * inv, st.o[d][4 * x + 3] * inv);
                *reinterpret_cast<uint2*>(dst + 32 * d + 8 * x) = y;
            }
}

// ---- prompts: K and V straight from bf16 rows ------------------------------------
template <int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void prompt_tile_kernel(PromptArgs a, int slots) {
    using C = TileShape_<DP>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t tile_smem[];
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), h = lane >> 5, l32 = lane & 31;
    const int G = a.Hq / a.H;
    // The tiles of prompt b have the slots from floor(cu[b] G / 128) + b on (some stay empty): which prompt a slot
    // belongs to takes one comparison per prompt.  Late tiles, the longest, go first; heads go round-robin over the
    // XCDs, so that a KV head's tiles share an L2.
    const int head = blockIdx.x % a.H, slot = slots - 1 - (int)(blockIdx.x / a.H);
    int b = -1, first = 0, n = 0;
    for (int x = 0; x < a.B; x += 64) {
        const int y = x + lane;
        int lo, rows;
        rows_of(a.cu, a.T, a.B, min(y, a.B - 1), &lo, &rows);
        const uint64_t votes = __ballot(y < a.B && (int64_t)lo * G / C::kRows + y <= slot);
        if (votes) {
            const int last = 63 - __builtin_clzll(votes);
            b = x + last;
            first = __builtin_amdgcn_readlane(lo, last);
            n = __builtin_amdgcn_readlane(rows, last);
        }
        if (votes != ~0ull) break;
    }
    if (b < 0) return;
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
    const uint16_t *k_at[C::kLoads], *v_at[C::kLoads];                          // of the next tile to load
    int k_part[C::kLoads], v_part[C::kLoads];
#pragma unroll
    for (int x = 0; x < C::kLoads; ++x) {
        const int r = (4 * x + w) * kPer + ld_key;
        const int ck = ld_slot ^ tile_k_swizzle<DP>(r), cv = ld_slot ^ tile_v_swizzle<DP>(r);
        k_part[x] = ck < chunks ? ck * 8 : -1;                                 // (past the head's end: not loaded, 0)
        v_part[x] = cv < chunks ? cv * 8 : 0;                                  // (past the head's end: any, not stored)
        k_at[x] = k_rows + r * a.ld_k + k_part[x];
        v_at[x] = v_rows + r * a.ld_v + v_part[x];
    }
    const int64_t k_step = C::kKeys * a.ld_k, v_step = C::kKeys * a.ld_v;
    // Keys' columns past the head's end stay 0: a key's infinity there times the queries' 0 would be NaN.
    const bool whole = a.D == DP;
    if (!whole) {
        for (int x = tid * 16; x < C::kTile; x += 256 * 16) {
            *reinterpret_cast<u32x4_t*>(tile_smem + x) = u32x4_t{0, 0, 0, 0};
            *reinterpret_cast<u32x4_t*>(tile_smem + 2 * C::kTile + x) = u32x4_t{0, 0, 0, 0};
        }
        __syncthreads();
    }
    const auto stage = [&](int t) {
        const uint32_t to = smem + (t & 1) * 2 * C::kTile;
        if ((t + 1) * C::kKeys > n) {                                          // past the end: the last key again
#pragma unroll
            for (int x = 0; x < C::kLoads; ++x) {
                const int64_t key = min(t * C::kKeys + (4 * x + w) * kPer + ld_key, n - 1);
                k_at[x] = k_rows + key * a.ld_k + k_part[x];
                v_at[x] = v_rows + key * a.ld_v + v_part[x];
            }
        }
#pragma unroll
        for (int x = 0; x < C::kLoads; ++x) {
            if (whole || k_part[x] >= 0) load_lds16(k_at[x], to + (4 * x + w) * 1024);
            load_lds16(v_at[x], to + C::kTile + (4 * x + w) * 1024);
            k_at[x] += k_step;
            v_at[x] += v_step;
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
    const bool both = first_token < kFewKeys;
    for (int t = 0; t < tiles; ++t) {
        if (t + 1 < tiles) stage(t + 1);
        const uint32_t kt = smem + (t & 1) * 2 * C::kTile;
        const int k0 = t * C::kKeys;
        uint8_t* const values = tile_smem + (t & 1) * 2 * C::kTile + C::kTile;
        if ((both || k0 + C::kKeys - 1 > first_token) && __syncthreads_or(wild_part<DP>(values))) {
            mark_tile(st, kt + C::kTile, first_keys(i + 1 - k0));
            __syncthreads();
            clean_part<DP>(values);
            __syncthreads();
        }
        if (k0 <= wave_last)
            attend_tile<DP, false>(st, q, kt, kt + C::kTile, first_keys(i + 1 - k0), k0 + C::kKeys - 1 <= wave_first, c2,
                                   false, both, nullptr, nullptr);
        wait_loads<0>();
        __syncthreads();
    }
    end_rows(st);
    if (there) store_rows(st, a.out + (int64_t)(first + i) * a.ld_out + (int64_t)(head * G + g) * a.D, a.D, 1.0f);
}

// ---- new rows over the paged FP8 cache --------------------------------------------
// Work: attn_line.hpp; a unit is (sequence, 32 W rows, one KV head), a step 64 keys.  The codes of the next tile
// are loaded to registers while a tile is attended to, and written to LDS as bf16 (exact) after it; the table entries of
// the tile after that travel meanwhile.  PT: one scale for the keys and one for the values.
// A wave's rows of a part leave through its corner of LDS, so that a store instruction writes whole rows (stored by
// 16 bytes of 32 rows each, a part took 22 us in place of 10): quads (four channels) of row r lie at slot
// quad ^ r, which spreads a column of them over the banks.
template <int DP>
struct RowBox {
    static constexpr int kQuads = DP / 4;
    static __device__ __forceinline__ int at(int row, int quad) { return row * kQuads + (quad ^ (row & (kQuads - 1))); }
    // the sums of `rows` rows to a part (through to memory)
    static __device__ __forceinline__ void store_part(const f32x4_t* box, float* to, int rows) {
        const int lane = threadIdx.x & 63;
        const float2* const pairs = reinterpret_cast<const float2*>(box);
        uint64_t* const dst = reinterpret_cast<uint64_t*>(to);
#pragma unroll 4
        for (int x = lane; x < rows * (DP / 2); x += 64) {
            const int r = x / (DP / 2), c = x % (DP / 2);
            const float2 v = pairs[2 * at(r, c >> 1) + (c & 1)];
            __hip_atomic_store(dst + x, two_floats(v.x, v.y), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
};

template <int DP>
constexpr int kTileWaves = DP == 128 ? 8 : 4;                // of a paged tile's workgroup, 32 rows each
constexpr int kTileCell = 8;                                 // steps that are worth a join of a whole tile's rows

template <int DP>
struct PagedTileShape {
    static constexpr int kScales = 4 * TileShape_<DP>::kTile;                  // two tiles' 64 + 64 scales and masks
    static constexpr int kLds = kScales + 2 * (512 + 16);
};

template <int DP, bool PT>
__global__ __launch_bounds__(64 * kTileWaves<DP>, DP == 256 ? 1 : 2) void paged_tile_kernel(PagedArgs a, float* part, unsigned int* tickets,
                                                                            int groups, int extra) {
    using C = TileShape_<DP>;
    constexpr int kThreads = 64 * kTileWaves<DP>, kRows = 32 * kTileWaves<DP>;
    extern __shared__ __attribute__((aligned(1024))) uint8_t tile_smem[];
    __shared__ LineShared<kThreads> sh;
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), h = lane >> 5, l32 = lane & 31;
    const int G = a.Hq / a.H;
    Line<kThreads, kRows, C::kKeys, kTileCell> line;
    if (!line.begin(a, sh, 1, groups, extra)) return;

    const uint32_t smem = uniform((int)lds_at(tile_smem));
    float* const scales = reinterpret_cast<float*>(tile_smem + PagedTileShape<DP>::kScales);      // [2][128]
    uint64_t* const masks = reinterpret_cast<uint64_t*>(scales + 256);                            // [2]
    // loads: 16 codes of key tid/kChunks + x kKeys16; table entries of those keys, and of the key whose scale this is
    constexpr int kChunks = DP / 16, kPer = kThreads / kChunks, NL = 64 / kPer;
    const int ld_row = tid / kChunks, ld_chunk = tid % kChunks, sc_key = tid & 63;
    // (rows 1 and 2 of each four change places: an LDS cycle serves lanes l and l + 16, whose chunks then differ)
    const int ld_key = DP == 128 ? (ld_row & ~3) | ((ld_row & 1) << 1) | ((ld_row >> 1) & 1) : ld_row;
    const int src_chunk = ld_chunk * 16 < a.D ? ld_chunk * 16 : 0;             // (past the head's end: any; queries are 0)
    // (a page has less than 4 GiB of codes)
    const int bs = a.block_size, step_q = C::kKeys / bs, step_r = C::kKeys % bs;
    const uint32_t row_bytes = a.H * a.D, page_bytes = bs * row_bytes, page_rows = bs * a.H;
    const int last_block = max(a.max_len / bs - 1, 0);
    // (as scalars of their own: a loop that reads one field of the arguments keeps, or reloads, eight)
    const uint32_t num_blocks = uniform(a.num_blocks);
    const int heads = uniform(a.H);
    const float* const scale_from = tid & 64 ? a.v_scale : a.k_scale;
    const float c2 = a.scale * 1.4426950408889634f * (PT ? a.k_scale[0] : 1.0f);
    const bool odd_c2 = PT && uniform(!(c2 > 0.0f && c2 < INFINITY));

    while (line.next(a, sh)) {
        const int n = line.n, L = line.L, first = line.first, head = line.hg;
        const int64_t R = (int64_t)n * G, row0 = (int64_t)line.rt * kRows;
        // the rows
        const int64_t row = row0 + 32 * w + l32;
        const bool there = row < R;
        const int i = there ? (int)(row / G) : 0, g = there ? (int)(row - (int64_t)i * G) : 0;
        const uint16_t* const src = a.q + (int64_t)(first + i) * a.ld_q + (int64_t)(head * G + g) * a.D;
        bf16x8_t q[C::KS];
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
            const int d = 16 * ks + 8 * h;
            u32x4_t v = *reinterpret_cast<const u32x4_t*>(src + min(d, a.D - 8));
            if (d >= a.D) v = u32x4_t{0, 0, 0, 0};
            q[ks] = __builtin_bit_cast(bf16x8_t, v);
        }
        // what they see: tokens up to lim, or a tree's; all of a tile up to some token; none past another
        const int lim = a.tree ? L - 1 : L - n + i;
        const uint64_t nodes = a.tree && there && i > 0 ? a.tree[(int64_t)line.b * a.N + i - 1] : 0;
        const auto first_of = [&](int64_t r) { return (int)min(r / G, (int64_t)n - 1); };
        const int all_see = a.tree ? L - a.N - 1 : L - n + uniform(first_of(row0));
        const int wave_all = a.tree ? all_see : L - n + uniform(first_of(row0 + 32 * w));
        const int wave_last = row0 + 32 * w >= R ? -1 : a.tree ? L - 1 : L - n + uniform(first_of(min(row0 + 32 * w + 31, R - 1)));
        const int last = a.tree ? L - 1 : L - n + uniform(first_of(min(row0 + kRows, R) - 1));
        const int count = min(line.count, (last >> 6) + 1 - line.s_in);        // (tiles that some row sees)
        const int is_tree = uniform(a.tree ? 1 : 0), node0 = uniform(L - a.N);
        const auto sees = [&](int k0) -> uint64_t {
            uint64_t m = first_keys(lim + 1 - k0);
            if (is_tree) {
                const int f = k0 - node0;                                       // node number of the tile's first key
                if (f >= 0) m &= f < 64 ? nodes >> f : 0;
                else if (f > -64) m &= nodes << -f | ((1ull << -f) - 1);
            }
            return m;
        };

        // ---- loads
        const int32_t* const table = a.max_len > 0 ? a.tables + (int64_t)line.b * a.ld_tables : a.kv_lens;
        int blk[NL + 1], off[NL + 1], page[NL + 1], in_page[NL + 1];
        int key0 = line.s_in * C::kKeys, code_key0 = key0;                     // first key of the tile to look up, to load
#pragma unroll
        for (int x = 0; x <= NL; ++x) {
            const int k = key0 + (x < NL ? ld_key + x * kPer : sc_key);
            blk[x] = k / bs;
            off[x] = k - blk[x] * bs;
        }
        const auto look_up = [&]() {
#pragma unroll
            for (int x = 0; x <= NL; ++x) {
                page[x] = table[min(blk[x], last_block)];
                in_page[x] = off[x];
                off[x] += step_r;
                blk[x] += step_q;
                if (off[x] >= bs) {
                    off[x] -= bs;
                    ++blk[x];
                }
            }
        };
        const uint32_t head_bytes = uniform(head * a.D);
        const uint8_t *const k_from = a.k_cache + src_chunk, *const v_from = a.v_cache + src_chunk;
        u32x4_t kc[NL], vc[NL];
        float scale = 0.0f;
        bool scale_there = false;
        uint64_t present = 0;                                                  // (wave 0) the keys that there are
        const auto load = [&]() {
#pragma unroll
            for (int x = 0; x <= NL; ++x) {
                const int k = code_key0 + (x < NL ? ld_key + x * kPer : sc_key);
                const bool ok = (k < L) & ((uint32_t)page[x] < num_blocks);
                const uint32_t pg = ok ? page[x] : 0, in = ok ? in_page[x] : 0;           // (not there: some row)
                if (x < NL) {
                    const uint64_t r = (uint64_t)pg * page_bytes + (in * row_bytes + head_bytes);
                    kc[x] = *reinterpret_cast<const u32x4_t*>(k_from + r);
                    vc[x] = *reinterpret_cast<const u32x4_t*>(v_from + r);
                } else {
                    const uint64_t r = (uint64_t)pg * page_rows + (in * heads + head);
                    present = __ballot(ok);
                    if constexpr (!PT) {
                        scale_there = ok;
                        scale = scale_from[r];
                    }
                }
            }
            code_key0 += C::kKeys;
        };
        const auto write = [&](int t) {
            uint8_t* const to = tile_smem + (t & 1) * 2 * C::kTile;
#pragma unroll
            for (int x = 0; x < NL; ++x) {
                const int r = ld_key + x * kPer;
                bf16x8_t* const krow = reinterpret_cast<bf16x8_t*>(to + r * C::kRowBytes);
                bf16x8_t* const vrow = reinterpret_cast<bf16x8_t*>(to + C::kTile + r * C::kRowBytes);
                const int fk = tile_k_swizzle<DP>(r), fv = tile_v_swizzle<DP>(r);
                krow[(2 * ld_chunk) ^ fk] = codes_to_bf16(kc[x][0], kc[x][1]);
                krow[(2 * ld_chunk + 1) ^ fk] = codes_to_bf16(kc[x][2], kc[x][3]);
                vrow[(2 * ld_chunk) ^ fv] = codes_to_bf16(vc[x][0], vc[x][1]);
                vrow[(2 * ld_chunk + 1) ^ fv] = codes_to_bf16(vc[x][2], vc[x][3]);
            }
            if (tid == 0) masks[t & 1] = present;
            if constexpr (!PT)
                if (tid < 128) scales[(t & 1) * 128 + tid] = scale_there ? (tid < 64 ? scale * c2 : scale) : 0.0f;
        };

        const bool both = all_see < kFewKeys;
        RowState<DP> st;
        begin_rows(st);
        if (count > 0) {
            look_up();
            load();
            if (count > 1) look_up();
            write(0);
            __syncthreads();
        }
        for (int t = 0; t < count; ++t) {
            if (t + 1 < count) load();
            if (t + 2 < count) look_up();
            const uint32_t kt = smem + (t & 1) * 2 * C::kTile;
            const int k0 = (line.s_in + t) * C::kKeys;
            const uint64_t mask = uniform((int64_t)masks[t & 1]);
            uint8_t* const values = tile_smem + (t & 1) * 2 * C::kTile + C::kTile;
            float* const sc = scales + (t & 1) * 128;
            if (mask != ~0ull || k0 + C::kKeys - 1 > all_see) {
                // (not there, or seen in part)
                const bool odd = !PT && tid < 64 && !(fabsf(sc[64 + tid]) < INFINITY);
                if (__syncthreads_or(mask != ~0ull || odd || wild_part<DP>(values))) {
                    settle_part<DP>(values, mask, PT ? nullptr : sc + 64);
                    __syncthreads();
                    if (odd) sc[64 + tid] = 0.0f;
                    const bool wild = __syncthreads_or(wild_part<DP>(values));
                    if (wild) {
                        mark_tile(st, kt + C::kTile, sees(k0) & mask);
                        __syncthreads();
                        clean_part<DP>(values);
                    }
                    __syncthreads();
                }
            }
            if (k0 <= wave_last) {
                const bool full = mask == ~0ull && k0 + C::kKeys - 1 <= wave_all;
                attend_tile<DP, !PT>(st, q, kt, kt + C::kTile, full ? 0 : sees(k0) & mask, full, c2, odd_c2, both, sc, sc + 64);
            }
            if (t + 1 < count) write(t + 1);
            __syncthreads();
        }
        end_rows(st);
        const float v_scale = PT ? a.v_scale[0] : 1.0f;
        if (line.whole()) {
            if (there) store_rows(st, a.out + (int64_t)(first + i) * a.ld_out + (int64_t)(head * G + g) * a.D, a.D, v_scale);
        } else {
            const Parts<kThreads, kRows, 1, DP, decltype(line)> parts(line, part, tickets, groups);
            // (a row that sees none of these keys has sums of 0, also under an infinite or NaN scale)
            const float part_scale = st.l == 0.0f ? 1.0f : v_scale;
            f32x4_t* const box = reinterpret_cast<f32x4_t*>(tile_smem + w * 32 * DP * 4);
#pragma unroll
            for (int d = 0; d < C::DB; ++d)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    box[RowBox<DP>::at(l32, 8 * d + 2 * x + h)] =
                        f32x4_t{st.o[d][4 * x], st.o[d][4 * x + 1], st.o[d][4 * x + 2], st.o[d][4 * x + 3]} * part_scale;
            RowBox<DP>::store_part(box, parts.sums(parts.me) + 32 * w * DP,
                                      (int)max(min(R - row0 - 32 * w, (int64_t)32), (int64_t)0));
            if (there && h == 0) parts.store_ml(32 * w + l32, st.m, st.l);
            parts.finish(a, line, sh);
        }
    }
}

}  // namespace

}  // namespace specfp8
