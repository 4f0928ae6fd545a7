// The position rotation of new queries and keys on the way into the paged FP8 cache.
//
// Mathematics.  Pair i of a head's first R channels turns by angle position * inv_freq[i].  The angle is taken in turns
// (position * inv_freq / 2 pi, its whole turns dropped) with the second factor in two parts of 64 bits, so that positions of
// 31 bits keep the accuracy of the first; sine and cosine of the rest, and the rotation, are fp32.  Keys are quantized from the
// rotated fp32 values, values as the plain cache write does it.
//
// A wave takes a token, or one of 2^log_parts parts of its rows (query heads, key heads, value heads): it evaluates the
// token's R/2 angles once, one a lane, and hands them round through its corner of LDS.  G lanes own a row, 2 VEC
// channels each: VEC of the lower and VEC of the upper half of the rotated channels, or 2 VEC side by side where
// neighbours turn together and where nothing turns.
//
// What bounds it: memory for many tokens (8191 of 32 + 2 x 8 heads of 128, keys as bf16 too: 43.6 us, 4.6 TB/s of 202 MB;
// a large copy runs at 5.1), a launch and three round trips one after the other for few (1 token 3.3 us, 320 4.7, of which
// 2.2 a launch): slot and position, then inv_freq, then, behind the exchange of angles, the rows.
// Not faster there: the next rows loaded under this one's arithmetic (47.5), more waves a SIMD (45.4 and 52.8), workgroups
// of 2 or 8 waves.  Stores past the caches gain 2 to 4 us here, and the attention that reads q next loses them.
#pragma once

#include "device_common.hpp"
#include "kernels.hpp"
#include "plan.hpp"

namespace specfp8 {

namespace {

constexpr int kRopeThreads = 256, kRopeWaves = kRopeThreads / kWave;
constexpr int kRopeMaxPairs = 256;           // of a head (D <= 512)
constexpr uint32_t kRopeMostBlocks = kRopeStep / kRopeWaves;

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

// The kernel's arguments, in no more bytes than a cheap launch has (a call that the host bounds takes 4.9 us with what
// surrounds it, 5.15 with 176 bytes): addresses of 48 bits, which is what the GPU has of them, strides in eights of elements.
enum RopePointer {
    kQ, kK, kV, kQOut, kKOut, kPositions, kInvFreq, kSlots, kKScale, kVScale, kKCache, kVCache,
    kRopePointers
};
struct RopeCall {
    uint32_t low[kRopePointers];
    uint16_t high[kRopePointers];
    uint32_t ld[kKOut + 1];
    uint32_t T;
    int64_t num_slots;
    uint16_t Hq, H;
    uint8_t D8, R8, per_tensor : 1, log_parts : 7;

    void set(RopePointer i, const void* p) {
        low[i] = (uint32_t)reinterpret_cast<uintptr_t>(p);
        high[i] = (uint16_t)(reinterpret_cast<uintptr_t>(p) >> 32);
    }
    template <class T>
    __device__ __forceinline__ T* at(RopePointer i) const {
        const uint64_t p = (uint64_t)high[i] << 32 | low[i];
        return (T*)(__attribute__((address_space(1))) T*)p;      // (of global memory)
    }
    __device__ __forceinline__ int64_t stride(RopePointer i) const { return (int64_t)ld[i] * 8; }
};
static_assert(sizeof(RopeCall) <= kCheapArgs, "a launch's cost");

// Angles of position `at`: cosine and sine of pair p at cs[p].  inv_freq / 2 pi is held in two parts and the product's whole
// turns are taken off inside a fused operation, so that the rest of a turn is off by some 2^-54 turns at every position (with
// one part by 2^-51 of the whole angle: twice the error of sine and cosine in fp32 at 31 bits).
__device__ __forceinline__ void rope_angles(int at, const double* inv_freq, int pairs, float2* cs) {
    for (int p = threadIdx.x & (kWave - 1); p < pairs; p += kWave) {
        constexpr double turn = 0.15915494309189535, rest_of_turn = -9.839338337591243e-18;       // 1 / 2 pi
        const double f = inv_freq[p], step = f * turn, rest = fma(f, rest_of_turn, fma(f, turn, -step));
        const double whole = rint(at * step);
        float s, c;
        sincospif(2.0f * (float)fma((double)at, rest, fma((double)at, step, -whole)), &s, &c);
        cs[p] = float2{c, s};
    }
}

template <int VEC, int G, bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rope_kv_write_kernel(RopeCall a) {
    __shared__ float2 angles[kRopeWaves][kRopeMaxPairs];
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    const int j = lane % G, sub = lane / G;
    const int Hq = a.Hq, H = a.H, D = 8 * a.D8, R = 8 * a.R8, rows = Hq + 2 * H, step = (kWave / G) << a.log_parts;
    const bool turns = 2 * VEC * j < R, mine = 2 * VEC * j < D;
    for (uint32_t item = blockIdx.x * kRopeWaves + w; item < a.T << a.log_parts; item += kRopeMostBlocks * kRopeWaves) {
        const int64_t t = item >> a.log_parts;
        const int part = (int)(item & ((1u << a.log_parts) - 1));
        const int64_t slot = a.at<const int64_t>(kSlots)[t];
        const bool stored = slot >= 0 && slot < a.num_slots;
        rope_angles(a.at<const int32_t>(kPositions)[t], a.at<const double>(kInvFreq), R / 2, angles[w]);
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
        const uint16_t* const q_in = a.at<const uint16_t>(kQ) + t * a.stride(kQ);
        const uint16_t* const k_in = a.at<const uint16_t>(kK) + t * a.stride(kK);
        const uint16_t* const v_in = a.at<const uint16_t>(kV) + t * a.stride(kV);
        uint16_t* const q_out = a.at<uint16_t>(kQOut) + t * a.stride(kQOut);
        uint16_t* const k_out = a.at<uint16_t>(kKOut);
        uint16_t* const k_row = k_out + t * a.stride(kKOut);
        for (int r0 = part * (kWave / G); r0 < rows; r0 += step) {
            const int r = r0 + sub;
            const bool live = mine && r < rows;
            const int kind = r < Hq ? 0 : r < Hq + H ? 1 : 2;                  // query, key, value
            const int head = kind == 0 ? r : kind == 1 ? r - Hq : r - Hq - H;
            const bool halves = !INTERLEAVED && turns && kind != 2;
            const int lo = halves ? VEC * j : 2 * VEC * j, hi = halves ? R / 2 + VEC * j : lo + VEC;
            float v[2 * VEC];
#pragma unroll
            for (int i = 0; i < 2 * VEC; ++i) v[i] = 0.0f;
            if (live) {
                const uint16_t* const src = (kind == 0 ? q_in : kind == 1 ? k_in : v_in) + (int64_t)head * D;
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
                if (kind == 0 || k_out) {
                    uint16_t* const dst = (kind == 0 ? q_out : k_row) + (int64_t)head * D;
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
            if (!stored || r0 + kWave / G <= Hq) continue;                   // (the same in all lanes)
            float amax = 0.0f;
#pragma unroll
            for (int i = 0; i < 2 * VEC; ++i) amax = fmaxf(amax, fabsf(v[i]));
#pragma unroll
            for (int o = G / 2; o >= 1; o /= 2) amax = fmaxf(amax, __shfl_xor(amax, o));
            if (kind == 0 || !live) continue;
            float* const scale = kind == 1 ? a.at<float>(kKScale) : a.at<float>(kVScale);
            const int64_t at = slot * H + head;
            float sc;
            if (a.per_tensor) {
                sc = scale[0];
            } else {
                sc = fmaxf((float)((double)amax / 448.0), 0x1p-100f);
                if (j == 0) scale[at] = sc;
            }
            const float inv = (float)(1.0 / (double)sc);
            uint8_t* const dst = (kind == 1 ? a.at<uint8_t>(kKCache) : a.at<uint8_t>(kVCache)) + at * D;
#pragma unroll
            for (int i = 0; i < 2 * VEC; ++i) v[i] *= inv;
            if constexpr (VEC == 8) {
                *reinterpret_cast<uint2*>(dst + lo) = uint2{e4m3x4(v[0], v[1], v[2], v[3]), e4m3x4(v[4], v[5], v[6], v[7])};
                *reinterpret_cast<uint2*>(dst + hi) =
                    uint2{e4m3x4(v[8], v[9], v[10], v[11]), e4m3x4(v[12], v[13], v[14], v[15])};
            } else {
                *reinterpret_cast<uint32_t*>(dst + lo) = e4m3x4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<uint32_t*>(dst + hi) = e4m3x4(v[4], v[5], v[6], v[7]);
            }
        }
    }
}

template <int VEC, int G>
void launch_rope_rows(const RopeCall& a, bool interleaved, unsigned blocks, hipStream_t stream) {
    if (interleaved)
        hipLaunchKernelGGL((rope_kv_write_kernel<VEC, G, true>), dim3(blocks), dim3(kRopeThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((rope_kv_write_kernel<VEC, G, false>), dim3(blocks), dim3(kRopeThreads), 0, stream, a);
}

}  // namespace

hipError_t launch_rope_kv_write(const RopeArgs& a, bool interleaved, hipStream_t stream) {
    const bool wide = a.D % 16 == 0 && a.R % 16 == 0;          // 16-byte loads of both halves
    const int vec = wide ? 8 : 4;
    int g = 1;
    while (2 * vec * g < a.D) g *= 2;
    const int log_parts = rope_log_parts(a.T, a.Hq, a.H, g);
    RopeCall c;
    const int64_t strides[] = {a.ld_q, a.ld_k, a.ld_v, a.ld_q_out, a.ld_k_out};
    for (int i = 0; i <= kKOut; ++i) c.ld[i] = (uint32_t)(strides[i] / 8);
    c.num_slots = a.num_slots;
    c.Hq = (uint16_t)a.Hq;
    c.H = (uint16_t)a.H;
    c.D8 = (uint8_t)(a.D / 8);
    c.R8 = (uint8_t)(a.R / 8);
    c.per_tensor = a.per_tensor != 0;
    c.log_parts = log_parts;
    c.T = (uint32_t)a.T;
    c.set(kQ, a.q);
    c.set(kK, a.k);
    c.set(kV, a.v);
    c.set(kQOut, a.q_out);
    c.set(kKOut, a.k_out);
    c.set(kPositions, a.positions);
    c.set(kInvFreq, a.inv_freq);
    c.set(kSlots, a.slot);
    c.set(kKScale, a.k_scale);
    c.set(kVScale, a.v_scale);
    c.set(kKCache, a.k_cache);
    c.set(kVCache, a.v_cache);
    const uint32_t items = c.T << log_parts;
    uint32_t blocks = (items + kRopeWaves - 1) / kRopeWaves;
    if (blocks > kRopeMostBlocks) blocks = kRopeMostBlocks;
#define SPEC_ROPE_CASE(V, N)                                    \
    case N:                                                     \
        launch_rope_rows<V, N>(c, interleaved, blocks, stream); \
        break;
    if (wide) {
        switch (g) {
            SPEC_ROPE_CASE(8, 1)
            SPEC_ROPE_CASE(8, 2)
            SPEC_ROPE_CASE(8, 4)
            SPEC_ROPE_CASE(8, 8)
            SPEC_ROPE_CASE(8, 16)
            default:
                launch_rope_rows<8, 32>(c, interleaved, blocks, stream);
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
                launch_rope_rows<4, 64>(c, interleaved, blocks, stream);
        }
    }
#undef SPEC_ROPE_CASE
    return hipGetLastError();
}

}  // namespace specfp8
