// FP8 KV-cache write: the new tokens' key and value heads, quantized to E4M3
// and scattered to their cache slots (section 3.2: an FP8 KV cache holds half
// the bytes of a bf16 one).
//
// The cache is slot-major, [num_slots][H][D] codes, which is the paged layout
// [blocks][block_size][H][D] for any block size (slot = block * block_size +
// offset).  One (token, head) row of D values is owned by a group of G lanes
// (G = D/8 rounded up to a power of two, at most 64): every lane holds 8 values
// from one 16-byte load, the group reduces max|v| with lane exchanges inside
// the wave, and each lane writes its 8 codes as one 8-byte store.  A wave
// therefore covers 64/G rows, a 256-thread block 256/G rows; blockIdx.y picks
// keys (0) or values (1).  Traffic is the algorithmic 2 bytes read and 1 byte
// written per element plus 4 bytes of scale per row in the per-row mode.
#include <algorithm>

#include "device_common.hpp"
#include "kernels.hpp"
#include "rope.hpp"

namespace specfp8 {

namespace {

constexpr int kKvThreads = 256;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

struct KvSide {
    const uint16_t* x;   // bf16 [T][ld_x]; head h of token t at x + t*ld_x + h*D
    int64_t ld_x;
    float* scale;        // per-row: [num_slots][H] (written); per-tensor: [1] (read)
    uint8_t* cache;      // [num_slots][H][D]
};

struct KvArgs {
    KvSide side[2];
    const int64_t* slot;
    int64_t T, H, D, num_slots;
    int per_tensor;
};

template <int G>
__global__ __launch_bounds__(kKvThreads) void kv_cache_write_kernel(KvArgs a) {
    const KvSide s = blockIdx.y ? a.side[1] : a.side[0];
    const int j = threadIdx.x % G;                                   // lane in the row's group
    const int64_t row = (int64_t)blockIdx.x * (kKvThreads / G) + threadIdx.x / G;
    const int64_t rows = a.T * a.H;
    int64_t t = 0, h = 0, slot = -1;
    if (row < rows) {
        t = row / a.H;
        h = row - t * a.H;
        slot = a.slot[t];
    }
    const bool live = slot >= 0 && slot < a.num_slots;
    const bool mine = live && (int64_t)j * 8 < a.D;
    float v[8];
    float amax = 0.0f;
    if (mine) {
        const uint4 p = *reinterpret_cast<const uint4*>(s.x + t * s.ld_x + h * a.D + (int64_t)j * 8);
        unpack8(p, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(v[e]));
    }
    // max over the G lanes of the row; every lane of the wave takes part
#pragma unroll
    for (int o = G / 2; o >= 1; o /= 2) amax = fmaxf(amax, __shfl_xor(amax, o));
    float sc;
    if (a.per_tensor) {
        sc = s.scale[0];
    } else {
        sc = fmaxf((float)((double)amax / 448.0), 0x1p-100f);
        if (live && j == 0) s.scale[slot * a.H + h] = sc;
    }
    if (!mine) return;
    const float inv = (float)(1.0 / (double)sc);
    uint2 o;
    o.x = e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
    o.y = e4m3x4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
    *reinterpret_cast<uint2*>(s.cache + (slot * a.H + h) * a.D + (int64_t)j * 8) = o;
}

// The reverse: the codes of cached tokens, decoded, scaled in fp32 and rounded once to bf16.  A token's
// heads lie one after the other on both sides, so P = H*D/8 lanes take a token, 8 codes each; a pass of the
// block covers 256/P tokens (P > 256: a token in several passes), and kReadTokens such passes are in flight
// at a time, slots first, then codes and scales.  Divisions are in 32 bits, outside the loops.  Traffic is 1
// byte read and 2 written per element and 4 of scale per row, and bounds it: 70001 tokens of 8 heads of 128
// take 77 us, 5.6 TB/s of the 435 MB (one lane per 8 codes that found its row by 64-bit divisions, one token
// in flight and cached stores: 100 us).
constexpr int kReadTokens = 4;

struct KvReadSide {
    uint16_t* x;
    int64_t ld_x;
    const float* scale;
    const uint8_t* cache;
};

struct KvReadArgs {
    KvReadSide side[2];
    const int64_t* slot;
    int64_t T, num_slots;
    uint32_t H, lanes, per_head;              // lanes: H*D/8 of a token; per_head: D/8
    int per_tensor;
};

__global__ __launch_bounds__(kKvThreads) void kv_cache_read_kernel(KvReadArgs a) {
    const KvReadSide s = blockIdx.y ? a.side[1] : a.side[0];
    const uint32_t P = a.lanes, tid = threadIdx.x;
    const uint32_t K = P < kKvThreads ? kKvThreads / P : 1, mine = P < kKvThreads ? tid / P : 0;
    if (mine >= K) return;
    const int64_t run = (int64_t)K * kReadTokens;
    for (int64_t t0 = blockIdx.x * run + mine; t0 < a.T; t0 += gridDim.x * run) {
        int64_t slot[kReadTokens];
#pragma unroll
        for (int u = 0; u < kReadTokens; ++u) {
            const int64_t t = t0 + (int64_t)u * K;
            slot[u] = t < a.T ? a.slot[t] : -1;
            if (slot[u] >= a.num_slots) slot[u] = -1;
        }
        for (uint32_t v = tid - mine * P; v < P; v += kKvThreads) {
            const uint32_t h = v / a.per_head;
            uint2 c[kReadTokens];
            float sc[kReadTokens];
#pragma unroll
            for (int u = 0; u < kReadTokens; ++u) {
                c[u] = uint2{0, 0};
                sc[u] = 0.0f;
                if (slot[u] >= 0) {
                    sc[u] = s.scale[a.per_tensor ? 0 : slot[u] * a.H + h];
                    c[u] = *reinterpret_cast<const uint2*>(s.cache + (slot[u] * P + v) * 8);
                }
            }
#pragma unroll
            for (int u = 0; u < kReadTokens; ++u) {
                const int64_t t = t0 + (int64_t)u * K;
                if (t >= a.T) break;
                u32x4_t o;
                o[0] = f32_to_bf16x2(__builtin_amdgcn_cvt_f32_fp8(c[u].x, 0) * sc[u], __builtin_amdgcn_cvt_f32_fp8(c[u].x, 1) * sc[u]);
                o[1] = f32_to_bf16x2(__builtin_amdgcn_cvt_f32_fp8(c[u].x, 2) * sc[u], __builtin_amdgcn_cvt_f32_fp8(c[u].x, 3) * sc[u]);
                o[2] = f32_to_bf16x2(__builtin_amdgcn_cvt_f32_fp8(c[u].y, 0) * sc[u], __builtin_amdgcn_cvt_f32_fp8(c[u].y, 1) * sc[u]);
                o[3] = f32_to_bf16x2(__builtin_amdgcn_cvt_f32_fp8(c[u].y, 2) * sc[u], __builtin_amdgcn_cvt_f32_fp8(c[u].y, 3) * sc[u]);
                __builtin_nontemporal_store(o, reinterpret_cast<u32x4_t*>(s.x + t * s.ld_x + (int64_t)v * 8));
            }
        }
    }
}

}  // namespace

hipError_t launch_kv_cache_read(const uint8_t* k_cache, const uint8_t* v_cache, const float* k_scale,
                                const float* v_scale, int per_tensor, const int64_t* slot_mapping, int64_t T,
                                int64_t H, int64_t D, int64_t num_slots, uint16_t* k, int64_t ld_k, uint16_t* v,
                                int64_t ld_v, hipStream_t stream) {
    KvReadArgs a;
    a.side[0] = KvReadSide{k, ld_k, k_scale, k_cache};
    a.side[1] = KvReadSide{v, ld_v, v_scale, v_cache};
    a.slot = slot_mapping;
    a.T = T;
    a.num_slots = num_slots;
    a.H = (uint32_t)H;
    a.lanes = (uint32_t)(H * D / 8);
    a.per_head = (uint32_t)(D / 8);
    a.per_tensor = per_tensor;
    const int64_t run = std::max<int64_t>(kKvThreads / a.lanes, 1) * kReadTokens;
    const int64_t blocks = std::min<int64_t>((T + run - 1) / run, (1 << 24) - 1);     // of fewer than 2^32 threads
    hipLaunchKernelGGL(kv_cache_read_kernel, dim3((unsigned)blocks, 2), dim3(kKvThreads), 0, stream, a);
    return hipGetLastError();
}

int64_t kv_group_lanes(int64_t D) {
    int64_t g = 1;
    while (g * 8 < D) g *= 2;
    return g;
}

hipError_t launch_kv_cache_write(const uint16_t* k, int64_t ld_k, const uint16_t* v, int64_t ld_v,
                                 const int64_t* slot_mapping, int64_t T, int64_t H, int64_t D,
                                 int64_t num_slots, int per_tensor, float* k_scale, float* v_scale,
                                 uint8_t* k_cache, uint8_t* v_cache, hipStream_t stream) {
    KvArgs a;
    a.side[0] = KvSide{k, ld_k, k_scale, k_cache};
    a.side[1] = KvSide{v, ld_v, v_scale, v_cache};
    a.slot = slot_mapping;
    a.T = T;
    a.H = H;
    a.D = D;
    a.num_slots = num_slots;
    a.per_tensor = per_tensor;
    const int64_t rows = T * H;
    const int64_t g = kv_group_lanes(D);
    const int64_t per_block = kKvThreads / g;
    dim3 grid((unsigned)((rows + per_block - 1) / per_block), 2), block(kKvThreads);
#define SPEC_KV_CASE(N)                                                                     \
    case N:                                                                                 \
        hipLaunchKernelGGL(kv_cache_write_kernel<N>, grid, block, 0, stream, a);            \
        break;
    switch (g) {
        SPEC_KV_CASE(1)
        SPEC_KV_CASE(2)
        SPEC_KV_CASE(4)
        SPEC_KV_CASE(8)
        SPEC_KV_CASE(16)
        SPEC_KV_CASE(32)
        default:
            hipLaunchKernelGGL(kv_cache_write_kernel<64>, grid, block, 0, stream, a);
    }
#undef SPEC_KV_CASE
    return hipGetLastError();
}

}  // namespace specfp8
