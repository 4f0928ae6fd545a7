// Root-mean-square norm of rows, with the residual's addition before it and E4M3 codes (or bf16) behind it.
//
// Mathematics.  h = x + residual in fp32 (two bf16 values: one rounding), y = (h w) r with
// r = 1 / sqrt(mean h^2 + eps).  Because the product with r is last and rounding keeps order, the row's
// largest |y| is fl32(max|h w| * r): the sum of squares and that maximum are reduced together, behind one barrier.
//
// One workgroup owns a row and keeps its sums in registers: every input is read once, every output written once.
#pragma once

#include "device_common.hpp"
#include "kernels.hpp"

namespace specfp8 {

namespace {

constexpr int kNormMaxThreads = 1024;

// Sum and maximum over the block, combined in a fixed order; `red` holds 32 floats and is not in use.
__device__ __forceinline__ void block_sum_max(float& sum, float& top, float* red) {
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave, nw = blockDim.x / kWave;
    sum = wave_sum(sum);
    top = wave_max(top);
    if (nw == 1) return;
    if (lane == 0) {
        red[w] = sum;
        red[16 + w] = top;
    }
    __syncthreads();
    sum = red[0];
    top = red[16];
    for (int i = 1; i < nw; ++i) {
        sum += red[i];
        top = fmaxf(top, red[16 + i]);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
    uint4 o;
    o.x = f32_to_bf16x2(v[0], v[1]);
    o.y = f32_to_bf16x2(v[2], v[3]);
    o.z = f32_to_bf16x2(v[4], v[5]);
    o.w = f32_to_bf16x2(v[6], v[7]);
    return o;
}

// NCH chunks of 8 channels per thread; chunk j of thread t is t + j * blockDim.x.
template <int NCH>
__global__ __launch_bounds__(kNormMaxThreads) void rms_norm_kernel(NormArgs a) {
    __shared__ float red[32], red2[32];
    const int64_t row = blockIdx.x;
    const int chunks = a.cols / 8, t = threadIdx.x, nt = blockDim.x;
    const uint16_t* const x = a.x + row * a.ld_x;
    uint4 raw[NCH], add[NCH], wt[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        raw[j] = add[j] = wt[j] = uint4{0, 0, 0, 0};
        if (t + j * nt < chunks) raw[j] = *reinterpret_cast<const uint4*>(x + (t + j * nt) * 8);
    }
    if (a.residual) {
        const uint16_t* const r = a.residual + row * a.ld_r;
#pragma unroll
        for (int j = 0; j < NCH; ++j)
            if (t + j * nt < chunks) add[j] = *reinterpret_cast<const uint4*>(r + (t + j * nt) * 8);
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j)
        if (t + j * nt < chunks) wt[j] = *reinterpret_cast<const uint4*>(a.weight + (t + j * nt) * 8);

    float h[NCH][8];
    float sum = 0.0f, top = 0.0f;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        float w[8];
        unpack8(raw[j], h[j]);
        if (a.residual) {
            float r[8];
            unpack8(add[j], r);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[j][e] += r[e];
        }
        unpack8(wt[j], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sum = fmaf(h[j][e], h[j][e], sum);
            top = fmaxf(top, fabsf(h[j][e] * w[e]));
        }
        if (a.sum && t + j * nt < chunks)
            *reinterpret_cast<uint4*>(a.sum + row * a.ld_sum + (t + j * nt) * 8) = pack8(h[j]);
    }
    block_sum_max(sum, top, red);
    const float cols = (float)a.cols;
    float r = 1.0f / sqrtf(sum / cols + a.eps);
    bool wild = false;                       // an infinite or NaN sum: the row is NaN throughout
    if (sum < 0x1p126f && top < 0x1p126f) {
        top *= r;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            float w[8];
            unpack8(wt[j], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[j][e] = (h[j][e] * w[e]) * r;
        }
    } else {
        // Squares or products beyond fp32: squares of 2^-80 h (eps is nothing beside them), products with r first.
        float pre = 1.0f, none = 0.0f;
        if (!(sum < 0x1p126f)) {
            pre = 0x1p-80f;
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < NCH; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(h[j][e] * pre, h[j][e] * pre, sum);
            block_sum_max(sum, none, red2);
            wild = !(sum < INFINITY);
            r = 1.0f / sqrtf(sum / cols);
        }
        top = 0.0f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            float w[8];
            unpack8(wt[j], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[j][e] = ((h[j][e] * pre) * r) * w[e];
                top = fmaxf(top, fabsf(h[j][e]));
            }
        }
        __syncthreads();                     // the first use of red
        block_sum_max(none, top, red);
    }
    float inv = 1.0f;
    if (a.q) {
        float s;
        if (a.per_tensor) {
            s = a.scales[0];
        } else {
            s = wild ? 0x1p-100f : fmaxf((float)((double)top / 448.0), 0x1p-100f);
            if (t == 0) a.scales[row] = s;
        }
        inv = (float)(1.0 / (double)s);
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int c = t + j * nt;
        if (c >= chunks) continue;
        if (a.y) {
            uint4 o = pack8(h[j]);
            if (wild) o = uint4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
            *reinterpret_cast<uint4*>(a.y + row * a.ld_y + c * 8) = o;
        }
        if (a.q) {
            uint2 o;
            o.x = e4m3x4(h[j][0] * inv, h[j][1] * inv, h[j][2] * inv, h[j][3] * inv);
            o.y = e4m3x4(h[j][4] * inv, h[j][5] * inv, h[j][6] * inv, h[j][7] * inv);
            if (wild) o = uint2{0x7f7f7f7fu, 0x7f7f7f7fu};
            *reinterpret_cast<uint2*>(a.q + row * a.ld_q + c * 8) = o;
        }
    }
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream) {
    const int chunks = a.cols / 8;
    int threads = 256;
    while (threads < kNormMaxThreads && chunks > 8 * threads) threads *= 2;
    if (chunks < threads) threads = (chunks + kWave - 1) / kWave * kWave;
    const int64_t most = 1 << 21;            // rows of a launch (a grid's threads are counted in 32 bits)
    if (a.rows > most) {
        NormArgs part = a;
        for (int64_t first = 0; first < a.rows; first += most) {
            part.rows = a.rows - first < most ? a.rows - first : most;
            part.x = a.x + first * a.ld_x;
            if (a.residual) part.residual = a.residual + first * a.ld_r;
            if (a.sum) part.sum = a.sum + first * a.ld_sum;
            if (a.y) part.y = a.y + first * a.ld_y;
            if (a.q) part.q = a.q + first * a.ld_q;
            if (a.q && !a.per_tensor) part.scales = a.scales + first;
            const hipError_t e = launch_rms_norm(part, stream);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    const dim3 grid((unsigned)a.rows), block(threads);
#define SPEC_NORM_CASE(N)                                                               \
    case N:                                                                             \
        hipLaunchKernelGGL(rms_norm_kernel<N>, grid, block, 0, stream, a);              \
        break;
    switch ((chunks + threads - 1) / threads) {
        SPEC_NORM_CASE(1)
        SPEC_NORM_CASE(2)
        SPEC_NORM_CASE(3)
        SPEC_NORM_CASE(4)
        SPEC_NORM_CASE(5)
        SPEC_NORM_CASE(6)
        SPEC_NORM_CASE(7)
        default:
            hipLaunchKernelGGL(rms_norm_kernel<8>, grid, block, 0, stream, a);
    }
#undef SPEC_NORM_CASE
    return hipGetLastError();
}

}  // namespace specfp8
