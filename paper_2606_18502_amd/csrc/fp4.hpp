// Weights in 4 bits (OCP MXFP4: E2M1 codes, one E8M0 scale for 32 of them) and their products with a few rows of
// E4M3 activations.
//
// Mathematics.  y[m,n] = sa(m) sum_g 2^(e[n,g] - 127) sum_{k in g} a[m,k] w[n,k]: v_mfma_scale_f32_16x16x128_f8f6f4
// multiplies 16 x 128 codes of 4 bits by 128 x 16 of 8 and takes a scale byte for each row and 32 k with it, so
// weights go from memory to the matrix cores as they are.
//
// A lane group g = lane / 16 of the weights' operand holds k 32 g .. of a row; of the activations' operand k 16 g .. and
// 64 + 16 g .. of a column.  The order of groups in the sum is free: step j of a stretch of 512 takes group 4 g + j from
// lane group g, so that a lane's weights of four steps are 64 bytes side by side and their scales one dword, which the
// steps pick their byte from.
#pragma once

#include "device_common.hpp"
#include "kernels.hpp"

namespace specfp8 {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kFp4Group = 32;

// ---- quantize: four lanes a group, 8 values each ----------------------------
// e is the exponent of the group's largest magnitude, rounded to E2M1's one bit after the point, less 2: that
// value becomes 4 or 6 (a scale from the unrounded one would cut 7 and more down to 6).
__global__ __launch_bounds__(256) void fp4_quantize_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t cols,
                                                           int64_t ld_x, uint8_t* __restrict__ q, int64_t ld_q,
                                                           uint8_t* __restrict__ scales, int64_t ld_s) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;              // chunk of 8 in the row
    if (c >= cols / 8) return;                                              // (whole groups leave: cols % 32 == 0)
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const uint4 v = *reinterpret_cast<const uint4*>(x + row * ld_x + c * 8);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        int top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max((int)(w[i] & 0x7fffu), (int)((w[i] >> 16) & 0x7fffu)));
        top = max(top, dpp_mov<0xB1>(top));
        top = max(top, dpp_mov<0x4E>(top));
        const int e = min(max(((top + 31 + ((top >> 6) & 1)) >> 7) - 2, 27), 252);      // with its bias of 127
        const float s = __uint_as_float((uint32_t)e << 23);
        uint32_t o = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
            const uint32_t two = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, lo, hi, s, 0);
            o |= (two & 0xffu) << (8 * i);
        }
        *reinterpret_cast<uint32_t*>(q + row * ld_q + c * 4) = o;
        if ((c & 3) == 0) scales[row * ld_s + c / 4] = (uint8_t)e;
    }
}

// ---- the product -------------------------------------------------------------
constexpr int kFp4Waves = 4;                                                // of a workgroup, each a share of K

template <int MT>
__global__ __launch_bounds__(64 * kFp4Waves) void gemm_fp4_kernel(Fp4Args a) {
    __shared__ f32x4_t box[kFp4Waves][MT][64];
    const int lane = threadIdx.x & 63, kw = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * 16 * MT;
    const int64_t n = min(n0 + r16, a.N - 1);
    const int groups = (int)(a.K / kFp4Group);
    const uint8_t* const w = a.w + n * a.ldw;
    const uint8_t* const ws = a.w_scale + n * a.ld_ws;
    f32x4_t acc[MT];
#pragma unroll
    for (int x = 0; x < MT; ++x) acc[x] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 16 * kw; s0 < groups; s0 += 16 * kFp4Waves) {
        const int first = s0 + 4 * g;                                       // this lane's groups: first .. first + 3
        uint32_t sc = 0x7f7f7f7fu;
        if (first + 4 <= groups) {
            __builtin_memcpy(&sc, ws + first, 4);
        } else {
            for (int j = 0; first + j < groups; ++j) sc = (sc & ~(0xffu << (8 * j))) | (uint32_t)ws[first + j] << (8 * j);
        }
        i32x8_t wv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 v = uint4{0, 0, 0, 0};
            if (first + j < groups) v = *reinterpret_cast<const uint4*>(w + (int64_t)(first + j) * 16);
            wv[j] = i32x8_t{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
        }
        i32x8_t av[MT][4];
#pragma unroll
        for (int x = 0; x < MT; ++x) {
            const int64_t m = m0 + 16 * x + r16;
            const uint8_t* const row = a.a + min(m, a.M - 1) * a.lda + 16 * (g & 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int lo = s0 + 4 * (g >> 1) + j, hi = lo + 8;
                uint4 u = uint4{0, 0, 0, 0}, v = uint4{0, 0, 0, 0};
                if (m < a.M && lo < groups) u = *reinterpret_cast<const uint4*>(row + (int64_t)lo * 32);
                if (m < a.M && hi < groups) v = *reinterpret_cast<const uint4*>(row + (int64_t)hi * 32);
                av[x][j] = i32x8_t{(int)u.x, (int)u.y, (int)u.z, (int)u.w, (int)v.x, (int)v.y, (int)v.z, (int)v.w};
            }
        }
#pragma unroll
        for (int x = 0; x < MT; ++x) {
            acc[x] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv[0], av[x][0], acc[x], 4, 0, 0, (int)sc, 0, 127);
            acc[x] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv[1], av[x][1], acc[x], 4, 0, 1, (int)sc, 0, 127);
            acc[x] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv[2], av[x][2], acc[x], 4, 0, 2, (int)sc, 0, 127);
            acc[x] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv[3], av[x][3], acc[x], 4, 0, 3, (int)sc, 0, 127);
        }
    }
#pragma unroll
    for (int x = 0; x < MT; ++x) box[kw][x][lane] = acc[x];
    __syncthreads();
    // a lane of the sum: 4 outputs n of one row m
    for (int x = kw; x < MT; x += kFp4Waves) {
        f32x4_t v = box[0][x][lane];
#pragma unroll
        for (int i = 1; i < kFp4Waves; ++i) v += box[i][x][lane];
        const int64_t m = m0 + 16 * x + r16, col = n0 + 4 * g;
        if (m >= a.M || col >= a.N) continue;
        v *= a.a_scale[a.per_tensor ? 0 : m];
        if (a.out_f32) {
            float* const y = reinterpret_cast<float*>(a.y) + m * a.ldy + col;
            if (col + 4 <= a.N) *reinterpret_cast<f32x4_t*>(y) = v;
            else
                for (int i = 0; col + i < a.N; ++i) y[i] = v[i];
        } else {
            uint16_t* const y = reinterpret_cast<uint16_t*>(a.y) + m * a.ldy + col;
            const uint2 o = uint2{f32_to_bf16x2(v[0], v[1]), f32_to_bf16x2(v[2], v[3])};
            if (col + 4 <= a.N) *reinterpret_cast<uint2*>(y) = o;
            else
                for (int i = 0; col + i < a.N; ++i) y[i] = (uint16_t)((i < 2 ? o.x : o.y) >> (16 * (i & 1)));
        }
    }
}

}  // namespace

hipError_t launch_fp4_quantize(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld_x, uint8_t* q, int64_t ld_q,
                               uint8_t* scales, int64_t ld_s, hipStream_t stream) {
    const dim3 grid((unsigned)((cols / 8 + 255) / 256), (unsigned)(rows < 65535 ? rows : 65535));
    hipLaunchKernelGGL(fp4_quantize_kernel, grid, dim3(256), 0, stream, x, rows, cols, ld_x, q, ld_q, scales, ld_s);
    return hipGetLastError();
}

hipError_t launch_gemm_fp4(const Fp4Args& a, hipStream_t stream) {
    const int mt = a.M <= 16 ? 1 : a.M <= 32 ? 2 : 4;
    const dim3 grid((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 16 * mt - 1) / (16 * mt))), block(64 * kFp4Waves);
    if (mt == 1)
        hipLaunchKernelGGL(gemm_fp4_kernel<1>, grid, block, 0, stream, a);
    else if (mt == 2)
        hipLaunchKernelGGL(gemm_fp4_kernel<2>, grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL(gemm_fp4_kernel<4>, grid, block, 0, stream, a);
    return hipGetLastError();
}

}  // namespace specfp8
