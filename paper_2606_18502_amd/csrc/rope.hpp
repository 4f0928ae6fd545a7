// The position rotation of new queries and keys on the way into the paged FP8 cache.
//
// Mathematics.  Pair i of a head's first R channels turns by angle position * inv_freq[i].  The angle is taken in
// 64 bits and in turns (position * inv_freq / 2 pi, its whole turns dropped), so that positions far into a context keep
// the accuracy of the first; sine and cosine of the rest, and the rotation, are fp32.  Keys are quantized from the
// rotated fp32 values, values as the plain cache write does it.
//
// A wave takes a token, or one of 2^log_parts parts of its rows (query heads, key heads, value heads): it evaluates the
// token's R/2 angles once, one a lane, and hands them round through its corner of LDS.  G lanes own a row, 2 VEC
// channels each: VEC of the lower and VEC of the upper half of the rotated channels, or 2 VEC side by side where
// neighbours turn together and where nothing turns.
//
// What bounds it: memory for many tokens (8191 of 32 + 2 x 8 heads of 128, keys as bf16 too: 44.4 us, 4.5 TB/s of 202 MB;
// a large copy runs at 5.1), a launch and three round trips for few (1 token 3.5 us, 320 4.4, of which 2.2 a launch).
// Not faster there: the next rows loaded under this one's arithmetic (47.5), more waves a SIMD (45.4 and 52.8), workgroups of 2 or
// 8 waves.  Stores past the caches gain 2 to 4 us here, and the attention that reads q next loses them.
#pragma once

#include "device_common.hpp"
#include "kernels.hpp"

namespace specfp8 {

namespace {

constexpr int kRopeThreads = 256, kRopeWaves = kRopeThreads / kWave;
constexpr int kRopeMaxPairs = 256;           // of a head (D <= 512)

// VEC (4 or 8) bf16 values
template <int VEC>
struct RopeChunk {
    uint32_t w[VEC / 2];
    __device__ __forceinline__ void load(const uint16_t* p) {
        if constexpr (VEC == 8) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(p);
        else *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
    }
    __device__ __forceinline__ void store(uint16_t* p) const {
        if constexpr (VEC == 8) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(w);
        else *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(w);
    }
};

// Angles of position `at`: cosine and sine of pair p at cs[p].
__device__ __forceinline__ void rope_angles(int at, const double* inv_freq, int pairs, float2* cs) {
    for (int p = threadIdx.x & (kWave - 1); p < pairs; p += kWave) {
        const double turns = (double)at * (inv_freq[p] * 0.15915494309189533577);
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        cs[p] = float2{c, s};
    }
}

template <int VEC, int G, bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rope_kv_write_kernel(RopeArgs a) {
    __shared__ float2 angles[kRopeWaves][kRopeMaxPairs];
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    const int j = lane % G, sub = lane / G;
    const int rows = a.Hq + 2 * a.H, D = a.D, step = (kWave / G) << a.log_parts;
    const bool turns = 2 * VEC * j < a.R, mine = 2 * VEC * j < D;
    const int64_t items = a.T << a.log_parts;
    for (int64_t item = (int64_t)blockIdx.x * kRopeWaves + w; item < items; item += (int64_t)gridDim.x * kRopeWaves) {
        const int64_t t = item >> a.log_parts;
        const int part = (int)(item & ((1 << a.log_parts) - 1));
        const int64_t slot = a.slot[t];
        const bool stored = slot >= 0 && slot < a.num_slots;
        rope_angles(a.positions[t], a.inv_freq, a.R / 2, angles[w]);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        float c[VEC], s[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float2 cs = turns ? angles[w][VEC * j + i] : float2{1.0f, 0.0f};
            c[i] = cs.x;
            s[i] = cs.y;
        }
        __builtin_amdgcn_wave_barrier();     // (the next token's angles are written after these reads)
        for (int r0 = part * (kWave / G); r0 < rows; r0 += step) {
            const int r = r0 + sub;
            const bool live = mine && r < rows;
            const int kind = r < a.Hq ? 0 : r < a.Hq + a.H ? 1 : 2;          // query, key, value
            const int head = kind == 0 ? r : kind == 1 ? r - a.Hq : r - a.Hq - a.H;
            const bool halves = !INTERLEAVED && turns && kind != 2;
            const int lo = halves ? VEC * j : 2 * VEC * j, hi = halves ? a.R / 2 + VEC * j : lo + VEC;
            float v[2 * VEC];
#pragma unroll
            for (int i = 0; i < 2 * VEC; ++i) v[i] = 0.0f;
            if (live) {
                const uint16_t* const src = (kind == 0 ? a.q + t * a.ld_q : kind == 1 ? a.k + t * a.ld_k : a.v + t * a.ld_v) +
                                            (int64_t)head * D;
                RopeChunk<VEC> x, y;
                x.load(src + lo);
                y.load(src + hi);
#pragma unroll
                for (int i = 0; i < VEC / 2; ++i) {
                    v[2 * i] = __uint_as_float(x.w[i] << 16);
                    v[2 * i + 1] = __uint_as_float(x.w[i] & 0xffff0000u);
                    v[VEC + 2 * i] = __uint_as_float(y.w[i] << 16);
                    v[VEC + 2 * i + 1] = __uint_as_float(y.w[i] & 0xffff0000u);
                }
            }
            if (kind != 2 && turns) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const int p = INTERLEAVED ? 2 * i : i, n = INTERLEAVED ? 2 * i + 1 : VEC + i;
                    const float x = v[p], y = v[n];
                    v[p] = fmaf(x, c[i], -(y * s[i]));
                    v[n] = fmaf(y, c[i], x * s[i]);
                }
            }
            if (kind != 2 && live) {
                uint16_t* const out = kind == 0 ? a.q_out : a.k_out;
                if (out) {
                    uint16_t* const dst = out + t * (kind == 0 ? a.ld_q_out : a.ld_k_out) + (int64_t)head * D;
                    RopeChunk<VEC> x, y;
#pragma unroll
                    for (int i = 0; i < VEC / 2; ++i) {
                        x.w[i] = f32_to_bf16x2(v[2 * i], v[2 * i + 1]);
                        y.w[i] = f32_to_bf16x2(v[VEC + 2 * i], v[VEC + 2 * i + 1]);
                    }
                    x.store(dst + lo);
                    y.store(dst + hi);
                }
            }
            if (!stored || r0 + kWave / G <= a.Hq) continue;                 // (the same in all lanes)
            float amax = 0.0f;
#pragma unroll
            for (int i = 0; i < 2 * VEC; ++i) amax = fmaxf(amax, fabsf(v[i]));
#pragma unroll
            for (int o = G / 2; o >= 1; o /= 2) amax = fmaxf(amax, __shfl_xor(amax, o));
            if (kind == 0 || !live) continue;
            float* const scale = kind == 1 ? a.k_scale : a.v_scale;
            const int64_t at = slot * a.H + head;
            float sc;
            if (a.per_tensor) {
                sc = scale[0];
            } else {
                sc = fmaxf((float)((double)amax / 448.0), 0x1p-100f);
                if (j == 0) scale[at] = sc;
            }
            const float inv = (float)(1.0 / (double)sc);
            uint8_t* const dst = (kind == 1 ? a.k_cache : a.v_cache) + at * D;
#pragma unroll
            for (int i = 0; i < 2 * VEC; ++i) v[i] *= inv;
            if constexpr (VEC == 8) {
                *reinterpret_cast<uint2*>(dst + lo) = uint2{e4m3x4(v[0], v[1], v[2], v[3]), e4m3x4(v[4], v[5], v[6], v[7])};
                *reinterpret_cast<uint2*>(dst + hi) = uint2{e4m3x4(v[8], v[9], v[10], v[11]), e4m3x4(v[12], v[13], v[14], v[15])};
            } else {
                *reinterpret_cast<uint32_t*>(dst + lo) = e4m3x4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<uint32_t*>(dst + hi) = e4m3x4(v[4], v[5], v[6], v[7]);
            }
        }
    }
}

template <int VEC, int G>
void launch_rope_rows(const RopeArgs& a, bool interleaved, int64_t blocks, hipStream_t stream) {
    if (interleaved)
        hipLaunchKernelGGL((rope_kv_write_kernel<VEC, G, true>), dim3((unsigned)blocks), dim3(kRopeThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((rope_kv_write_kernel<VEC, G, false>), dim3((unsigned)blocks), dim3(kRopeThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_rope_kv_write(const RopeArgs& given, bool interleaved, hipStream_t stream) {
    RopeArgs a = given;
    const bool wide = a.D % 16 == 0 && a.R % 16 == 0;          // 16-byte loads of both halves
    const int vec = wide ? 8 : 4;
    int g = 1;
    while (2 * vec * g < a.D) g *= 2;
    // Parts of a token while the waves hardly fill the chip, each with some rows of its own (1024 tokens in two parts 7.2 us;
    // 2048 in two 10.2, in one 10.9, but 2000 with heads of 256 12.1 and 10.5).
    const int64_t passes = ((int64_t)a.Hq + 2 * a.H) * g / kWave;
    a.log_parts = 0;
    while ((2LL << a.log_parts) <= passes && a.T << a.log_parts < 2048) ++a.log_parts;
    int64_t blocks = ((a.T << a.log_parts) + kRopeWaves - 1) / kRopeWaves;
    if (blocks > (1 << 24) - 1) blocks = (1 << 24) - 1;        // of fewer than 2^32 threads
#define SPEC_ROPE_CASE(V, N)                                   \
    case N:                                                    \
        launch_rope_rows<V, N>(a, interleaved, blocks, stream); \
        break;
    if (wide) {
        switch (g) {
            SPEC_ROPE_CASE(8, 1)
            SPEC_ROPE_CASE(8, 2)
            SPEC_ROPE_CASE(8, 4)
            SPEC_ROPE_CASE(8, 8)
            SPEC_ROPE_CASE(8, 16)
            default:
                launch_rope_rows<8, 32>(a, interleaved, blocks, stream);
        }
    } else {
        switch (g) {
            SPEC_ROPE_CASE(4, 1)
            SPEC_ROPE_CASE(4, 2)
            SPEC_ROPE_CASE(4, 4)
            SPEC_ROPE_CASE(4, 8)
            SPEC_ROPE_CASE(4, 16)
            SPEC_ROPE_CASE(4, 32)
            default:
                launch_rope_rows<4, 64>(a, interleaved, blocks, stream);
        }
    }
#undef SPEC_ROPE_CASE
    return hipGetLastError();
}

}  // namespace specfp8
