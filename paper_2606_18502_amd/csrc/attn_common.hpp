// What the attention kernels share: where a sequence's rows are, LDS loads
// and reads, lane exchanges.
#pragma once

#include "device_common.hpp"
#include "kernels.hpp"
#include "plan.hpp"

namespace specfp8 {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
#define SPEC_LDS __attribute__((address_space(3)))

constexpr float kLowest = -3.402823466e38f;   // a reference below every finite score
constexpr float kLazy = 8.0f;                 // powers of two that a score may exceed its row's reference by

// The rows of sequence b: first row and count (clamped into [0, T)).
__device__ __forceinline__ void rows_of(const int32_t* cu, int T, int B, int b, int* first, int* n) {
    if (!cu) {
        *n = T / B;
        *first = b * *n;
        return;
    }
    const int lo = min(max(cu[b], 0), T), hi = min(max(cu[b + 1], lo), T);
    *first = lo;
    *n = hi - lo;
}

// A value that is the same in all lanes, as a scalar.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return (int64_t)(((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32) | (uint32_t)uniform((int)v));
}

__device__ __forceinline__ uint32_t lds_at(const void* p) {
    return (uint32_t)(uintptr_t)(const SPEC_LDS void*)p;
}

// 16 (4) bytes per lane from its own address to LDS at `lds` + 16 (4) * lane.  Inline asm: the
// compiler would drain every load in flight before the next LDS read; the
// issuing code waits with explicit vmcnt counts instead.
__device__ __forceinline__ void load_lds16(const void* src, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void load_lds4(const void* src, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "{m0}"(lds) : "memory");
}

// Until at most N of this wave's vector memory operations are outstanding.
template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// This wave's LDS reads and writes are done.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Eight E4M3 codes as bf16 (exact).
__device__ __forceinline__ bf16x8_t codes_to_bf16(uint32_t lo, uint32_t hi) {
    u32x4_t r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    return __builtin_bit_cast(bf16x8_t, r);
}

// The NaN codes of four E4M3 bytes: 0x80 in each byte that is S.1111.111.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// Two bits as two bf16 values 0 or 1.
__device__ __forceinline__ uint32_t ones(uint32_t two) { return (two & 1u) * 0x3f80u | ((two >> 1) & 1u) * 0x3f800000u; }

// Maximum (sum) over the lanes l, l ^ 32, and over l, l ^ 16, l ^ 32, l ^ 48: the same value in each of them.
__device__ __forceinline__ float max_halves(float v) {
    const uint32_t x = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const uint32_t x = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_quarters(float v) {
    const uint32_t x = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float sum_quarters(float v) {
    const uint32_t x = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint64_t two_floats(float a, float b) {
    return (uint64_t)__float_as_uint(a) | ((uint64_t)__float_as_uint(b) << 32);
}

// Stores and loads that meet across XCDs without fences (the last arriver of a ticket reads what others stored).
__device__ __forceinline__ void store_agent(float* p, f32x4_t v) {
    uint64_t* q = reinterpret_cast<uint64_t*>(p);
    __hip_atomic_store(q, two_floats(v[0], v[1]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(q + 1, two_floats(v[2], v[3]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x4_t load_agent(const float* p) {
    uint64_t* q = reinterpret_cast<uint64_t*>(const_cast<float*>(p));
    const uint64_t a = __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint64_t b = __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    f32x4_t v;
    v[0] = __uint_as_float((uint32_t)a);
    v[1] = __uint_as_float((uint32_t)(a >> 32));
    v[2] = __uint_as_float((uint32_t)b);
    v[3] = __uint_as_float((uint32_t)(b >> 32));
    return v;
}

}  // namespace

}  // namespace specfp8
