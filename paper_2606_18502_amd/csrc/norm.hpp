// Root-mean-square norm of rows, with the residual's addition before it and E4M3 codes (or bf16) behind it.
//
// Mathematics.  h = x + residual in fp32 (two bf16 values: one rounding), y = (h w) r with
// r = 1 / sqrt(mean h^2 + eps).  Because the product with r is last and rounding keeps order, the row's
// largest |y| is fl32(max|h w| * r): the sum of squares and that maximum are reduced together, behind one barrier.
//
// One workgroup owns a row and keeps its sums in registers (rows of up to 32768 channels): every input is read once, every
// output written once.  What bounds it: memory for many rows (8191 x 4096 with residual and codes 41 us, 5.7 TB/s of
// 235 MB; a large copy runs at 5.1), a launch and two round trips for few (1 x 4096 2.6 us, of which 2.2 a launch).
// 1000 x 65536 take 126 us (3.6 TB/s of what has to move): read twice.  Rows whose squares or products exceed fp32 sum them
// scaled and take y from 64 bits; the test for them costs nothing that shows (320 x 4096 in a graph 3.85 us, without 3.86).
#pragma once

#include "device_common.hpp"
#include "kernels.hpp"

namespace specfp8 {

namespace {

constexpr int kNormMaxThreads = 1024;

// Sum and maximum over the block, combined in a fixed order; `red` holds 32 floats and is not in use.
__device__ __forceinline__ void block_sum_max(float& sum, float& top, float* red, int nw) {
    const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
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

// NCH > 0: NCH chunks of 8 channels per thread (chunk j of thread t is t + j * blockDim.x), loaded before any is used and
// kept.  NCH == 0: rows too wide for registers; every pass reads x, the residual and the weights again, and the sum is
// written in the last one, which may be where x or the residual lay.
template <int NCH>
__global__ __launch_bounds__(kNormMaxThreads) void rms_norm_kernel(NormArgs a) {
    __shared__ float red[32], red2[32];
    const int64_t row = blockIdx.x;
    const int chunks = a.cols / 8, t = threadIdx.x, nt = a.threads, nw = nt / kWave;
    const uint16_t *const x = a.x + row * a.ld_x, *const residual = a.residual ? a.residual + row * a.ld_r : nullptr;
    const auto load = [](const uint16_t* p, int64_t c) { return *reinterpret_cast<const uint4*>(p + c * 8); };
    // (past the caches: it is read when the layer's linears have run.  With 64 MB of other reads and its own behind it
    // 8191 x 4096 take 64.9 us, 67.1 through the caches; fewer rows the same.  Codes and values are read next: what their
    // stores gain so, their readers lose.)
    const auto store_sum = [&](int64_t c, const float (&h)[8]) {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        const uint4 o = pack8(h);
        __builtin_nontemporal_store(u32x4{o.x, o.y, o.z, o.w}, reinterpret_cast<u32x4*>(a.sum + row * a.ld_sum + c * 8));
    };
    const auto add = [&](const uint4& raw, const uint4& more, float (&h)[8]) {
        unpack8(raw, h);
        if (residual) {
            float r[8];
            unpack8(more, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] += r[e];
        }
    };
    float h[NCH > 0 ? NCH : 1][8];
    uint4 wt[NCH > 0 ? NCH : 1];
    if constexpr (NCH > 0) {
        uint4 raw[NCH], more[NCH];
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            raw[j] = more[j] = wt[j] = uint4{0, 0, 0, 0};
            if (t + j * nt < chunks) raw[j] = load(x, t + j * nt);
        }
        if (residual) {
#pragma unroll
            for (int j = 0; j < NCH; ++j)
                if (t + j * nt < chunks) more[j] = load(residual, t + j * nt);
        }
#pragma unroll
        for (int j = 0; j < NCH; ++j)
            if (t + j * nt < chunks) wt[j] = load(a.weight, t + j * nt);
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            add(raw[j], more[j], h[j]);
            if (a.sum && t + j * nt < chunks) store_sum(t + j * nt, h[j]);
        }
    }
    // f(chunk, its sums, its weights) for this thread's chunks (a chunk behind the row's end: zeros)
    const auto each = [&](auto f) {
        float w[8];
        if constexpr (NCH > 0) {
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                unpack8(wt[j], w);
                f(t + j * nt, h[j], w);
            }
        } else {
#pragma unroll 2
            for (int c = t; c < chunks; c += nt) {
                add(load(x, c), residual ? load(residual, c) : uint4{0, 0, 0, 0}, h[0]);
                unpack8(load(a.weight, c), w);
                f(c, h[0], w);
            }
        }
    };
    float sum = 0.0f, top = 0.0f;
    each([&](int, const float (&v)[8], const float (&w)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sum = fmaf(v[e], v[e], sum);
            top = fmaxf(top, fabsf(v[e] * w[e]));
        }
    });
    block_sum_max(sum, top, red, nw);
    const float cols = (float)a.cols;
    const bool fits = sum < 0x1p126f && a.eps < 0x1p126f;    // (and the mean with eps)
    const bool plain = fits && top < 0x1p126f;
    float r = 1.0f / sqrtf(sum / cols + a.eps), pre = 1.0f;
    bool wild = false;                       // an infinite or NaN sum: the row is NaN throughout
    const auto far = [&](float v, float w) { return (float)((double)v * w * ((double)r * pre)); };
    if (plain) {
        top *= r;
    } else {
        // Squares or products beyond fp32: squares of 2^-80 h (and eps 2^-160 beside their mean), y from 64 bits.
        float none = 0.0f;
        if (!fits) {
            pre = 0x1p-80f;
            sum = 0.0f;
            each([&](int, const float (&v)[8], const float (&)[8]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(v[e] * pre, v[e] * pre, sum);
            });
            block_sum_max(sum, none, red2, nw);
            wild = !(sum < INFINITY);
            r = 1.0f / sqrtf(sum / cols + a.eps * pre * pre);
        }
        top = none = 0.0f;
        each([&](int, const float (&v)[8], const float (&w)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(far(v[e], w[e])));
        });
        __syncthreads();                     // the first use of red
        block_sum_max(none, top, red, nw);
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
    const auto finish = [&](auto value) {
        each([&](int c, const float (&v)[8], const float (&w)[8]) {
            if (NCH > 0 && c >= chunks) return;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = value(v[e], w[e]);
            if (NCH == 0 && a.sum) store_sum(c, v);
            if (a.y) {
                uint4 o = pack8(y);
                if (wild) o = uint4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
                *reinterpret_cast<uint4*>(a.y + row * a.ld_y + (int64_t)c * 8) = o;
            }
            if (a.q) {
                uint2 o;
                o.x = e4m3x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
                o.y = e4m3x4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv);
                if (wild) o = uint2{0x7f7f7f7fu, 0x7f7f7f7fu};
                *reinterpret_cast<uint2*>(a.q + row * a.ld_q + (int64_t)c * 8) = o;
            }
        });
    };
    if (plain) finish([&](float v, float w) { return (v * w) * r; });
    else finish(far);
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& given, int64_t rows, hipStream_t stream) {
    NormArgs a = given;
    const int chunks = a.cols / 8;
    // One wave where two chunks a lane cover the row (no barrier), then up to four chunks a thread: 320 x 4096 4.1 us with
    // 256 threads, 4.8 with 128, 4.2 with 512; 1005 x 7176 8.9 with 256, 9.9 with 512; 2000 x 16384 44.1 with 512, 52.5
    // with 1024 (eight chunks in 256 threads spill: 79.6).
    int threads = chunks <= 2 * kWave ? kWave : 256;
    while (threads > kWave && threads < kNormMaxThreads && chunks > 4 * threads) threads *= 2;
    if (threads > kWave && chunks < threads) threads = (chunks + kWave - 1) / kWave * kWave;
    const int64_t most = 1 << 21;            // rows of a launch (a grid's threads are counted in 32 bits)
    a.threads = threads;
    for (int64_t first = 0; first < rows; first += most) {
        const dim3 grid((unsigned)(rows - first < most ? rows - first : most)), block(threads);
#define SPEC_NORM_CASE(N)                                                               \
    case N:                                                                             \
        hipLaunchKernelGGL(rms_norm_kernel<N>, grid, block, 0, stream, a);              \
        break;
        switch ((chunks + threads - 1) / threads) {
            SPEC_NORM_CASE(1)
            SPEC_NORM_CASE(2)
            SPEC_NORM_CASE(3)
            SPEC_NORM_CASE(4)
            default:
                hipLaunchKernelGGL(rms_norm_kernel<0>, grid, block, 0, stream, a);
        }
#undef SPEC_NORM_CASE
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || rows - first <= most) return e;
        a.x += most * a.ld_x;
        if (a.residual) a.residual += most * a.ld_r;
        if (a.sum) a.sum += most * a.ld_sum;
        if (a.y) a.y += most * a.ld_y;
        if (a.q) a.q += most * a.ld_q;
        if (a.q && !a.per_tensor) a.scales += most;
    }
    return hipSuccess;
}

}  // namespace specfp8
