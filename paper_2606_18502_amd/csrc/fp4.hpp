// Weights in 4 bits (OCP MXFP4: E2M1 codes, one E8M0 scale for 32 of them) and their products with a few rows of
// E4M3 activations.
//
// Mathematics.  y[m,n] = sa(m) sum_g 2^(e[n,g] - 127) sum_{k in g} a[m,k] w[n,k]: v_mfma_scale_f32_16x16x128_f8f6f4
// multiplies 16 x 128 codes of 4 bits by 128 x 16 of 8 and takes a scale byte for each row and 32 k with it, so
// weights go from memory to the matrix cores as they are.
//
// A lane group g = lane / 16 of the weights' operand holds k 32 g .. of a row and applies the scale byte that it
// brings to them; of the activations' operand k 16 g .. and 64 + 16 g .. of a column.
//
// What bounds it: W's bytes.  8 rows by 128256 x 4096 take 51.8 us (5.4 TB/s of 279 MB; a read of a large array 5.8).
// Smaller weights that were read a short while ago come from the Infinity Cache: 5 by 4096 x 14336 7.4 us, from memory 8.9;
// 1 by 6144 x 4096 4.7 and 5.9, of which 2.2 a launch.  With 64 rows A counts, too: every workgroup
// reads its rows of it (64 by 28672 x 4096 16.1 us, from memory 21.5, 62 MB of W; 64 by 4096 x 14336 12.0 and 16.6, 117 MB
// of A and 59 of W for 29 in memory), and from LDS each wave.  Operands straight from memory to registers took 94, 11.6, 5.9
// and 66 us for the first four (weights in the cache where they fit): 16 rows a load instruction in the matrix cores' order of lanes, and scales word by word.
#pragma once

#include <type_traits>
#include <utility>

#include "attn_common.hpp"
#include "kernels.hpp"
#include "plan.hpp"

namespace specfp8 {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

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
// MR rows of A (8, or a multiple of 16) and NT NW tiles of 16 rows of W a workgroup.  KW waves (or groups of NW waves, each
// with NT tiles of its own) share K, 128 at a time (a step), and stream their steps through rings of D stages of LDS: W and
// A go there without registers.  A step's operands are read from its stage under the products of the step before, and
// the stage is loaded anew.  Scales, a 32nd of the operands' count, go there some thousand k at a time in 16-byte pieces:
// a word a row and step, loaded with the stages, cost a fifth of 8 rows by 128256 x 4096.  Waves on their own wait for
// their own loads; groups meet at a barrier a step.  Two steps a stage (half the barriers) were within 5% at the shapes
// with many steps and slower where they left a ring of two.  Chunks of 16 bytes lie at slot c ^ f(row) of their row, so
// that the 16 lanes that an LDS cycle serves (lanes l and l + 16, l % 16 < 8) hit different banks.
template <int MR, int NT, int KW, int NW, int D>
struct Fp4Shape {
    static constexpr int MT = (MR + 15) / 16;                               // tiles of 16 rows of A
    static constexpr int kTiles = NT * NW, kThreads = 64 * KW * NW;
    static constexpr int kA = kTiles * 1024;                                // of a stage: W [16 NT NW][64], A [MR][128]
    static constexpr int kStage = kA + MR * 128;
    static constexpr int kLoadsA = MR / 8 / NW;                             // a wave's load instructions of a stage
    static constexpr int kLoads = NT + kLoadsA;
    static constexpr int kBox = KW > 1 ? KW * kTiles * MT * 1024 : 0;           // the waves' sums
    static constexpr int kScales = KW * D * kStage;                         // of kPanel steps: a word for each and row
    static constexpr int kPanel = fp4_panel(kTiles);
    static constexpr int kPieces = (4 * kTiles * kPanel + kThreads - 1) / kThreads;         // of 16 bytes of scales a thread
    static constexpr int lds(int64_t steps) {
        const int ring = kScales + 16 * kTiles * 4 * ((int)(steps < kPanel ? steps : kPanel) | 1);
        return ring > kBox ? ring : kBox;
    }
    static_assert(kScales + 64 * kTiles * (kPanel | 1) <= 160 * 1024 && kBox <= 160 * 1024, "a compute unit's LDS");
    static_assert(kPanel % KW == 0, "a wave's steps go on in the next panel");
    static_assert((NW == 1 || MR % (8 * NW) == 0) && D > 1, "a stage's loads are shared evenly");
    static_assert((D - 1) * kLoads < 64, "loads in flight are counted in 6 bits");
};
__device__ __forceinline__ int fp4_w_swizzle(int r) { return 2 * ((r >> 2) & 1); }
__device__ __forceinline__ int fp4_a_swizzle(int r) { return 2 * ((r >> 1) & 3); }

// Until the loads of at most `stages` stages of P each are outstanding.
template <int P, int MOST>
__device__ __forceinline__ void wait_stages(int stages) {
    if constexpr (MOST == 0) {
        wait_loads<0>();
    } else {
        if (stages >= MOST) wait_loads<P * MOST>();
        else wait_stages<P, MOST - 1>(stages);
    }
}

// The operands of a step's products.
template <int MT, int NT>
struct Fp4Operands {
    i32x8_t a[MT];
    u32x4_t w[NT];
    uint32_t scale[NT];
};

template <int MR, int NT, int KW, int NW, int D>
__global__ __launch_bounds__(64 * KW * NW) void gemm_fp4_kernel(Fp4Args a) {
    using C = Fp4Shape<MR, NT, KW, NW, D>;
    constexpr int MT = C::MT;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int lane = threadIdx.x & 63, wave = uniform((int)(threadIdx.x >> 6)), r16 = lane & 15, g = lane >> 4;
    const int kw = wave / NW, nw = wave % NW;
    // Workgroups go to the 8 XCDs in turn: those of further rows start so far into the columns that the ones that share
    // columns of W, but for the last few, share an XCD's L2, too (24 by 3000 x 4096 4.9 us without, 4.3 with; 256 by
    // 6000 x 14336 43.7, 38.3).
    const unsigned across = (unsigned)((a.N + 16 * C::kTiles - 1) / (16 * C::kTiles));
    unsigned tile = blockIdx.x + (across >= 8 ? across * blockIdx.y % 8 : 0);
    if (tile >= across) tile -= across;
    const int64_t first_n = (int64_t)tile * (16 * C::kTiles), n0 = first_n + 16 * NT * nw, m0 = (int64_t)blockIdx.y * MR;
    const int K = uniform((int)a.K), steps = K / 128;                       // whole ones
    uint8_t* const ring = smem + kw * (D * C::kStage);
    const uint32_t ring_at = uniform((int)lds_at(ring));
    // (a row that is not there reads the last one; its products are not stored)
    const uint8_t *w_from[NT], *a_from[C::kLoadsA];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = lane / 4;
        w_from[t] = a.w + min(n0 + 16 * t + r, a.N - 1) * a.ldw + 64 * kw + (((lane & 3) ^ fp4_w_swizzle(r)) << 4);
    }
#pragma unroll
    for (int x = 0; x < C::kLoadsA; ++x) {
        const int r = 8 * (x * NW + nw) + lane / 8;
        a_from[x] = a.a + min(m0 + r, a.M - 1) * a.lda + 128 * kw + (((lane & 7) ^ fp4_a_swizzle(r)) << 4);
    }
    uint32_t* const scales = reinterpret_cast<uint32_t*>(smem + C::kScales);
    const int stride = min(steps, C::kPanel) | 1;                           // words of a row, odd: rows in different banks

    f32x4_t acc[NT][MT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int x = 0; x < MT; ++x) acc[t][x] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const auto multiply = [&](int t, int x, const u32x4_t& w, const i32x8_t& av, uint32_t scale) {
        const i32x8_t wv = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
        acc[t][x] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv, av, acc[t][x], 4, 0, 0, (int)scale, 0, 127);
    };
    const auto operand = [](const u32x4_t& lo, const u32x4_t& hi) {
        return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    const int ar = MR == 8 ? r16 & 7 : r16;
    const int w_at = NT * nw * 1024 + r16 * 64 + ((g ^ fp4_w_swizzle(r16)) << 4);
    const int a_at = C::kA + ar * 128 + ((g ^ fp4_a_swizzle(ar)) << 4);
    for (int p0 = 0; p0 < steps; p0 += C::kPanel) {
        const int in_panel = min(steps - p0, C::kPanel);
        const int count = uniform((in_panel - kw + KW - 1) / KW);          // this wave's: kw, kw + KW, ..
        const auto load = [&](int slot) {    // the next one
            const uint32_t to = ring_at + slot * C::kStage;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                load_lds16(w_from[t], to + (NT * nw + t) * 1024);
                w_from[t] += 64 * KW;
            }
#pragma unroll
            for (int x = 0; x < C::kLoadsA; ++x) {
                load_lds16(a_from[x], to + C::kA + (x * NW + nw) * 1024);
                a_from[x] += 128 * KW;
            }
        };
        if (p0) {                            // the reads of the last panel's scales and stages
            wait_lds();
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < D; ++i)
            if (i < count) load(i);
        // The panel's scales, a word for each row and step, from rows of any address.
        {
            const int pieces = (in_panel + 3) / 4;
            u32x4_t v[C::kPieces];
#pragma unroll
            for (int x = 0; x < C::kPieces; ++x) {
                const int i = threadIdx.x + x * C::kThreads, row = i / pieces, c = i - row * pieces;
                if (row >= 16 * C::kTiles) continue;
                const uint8_t* const from = a.w_scale + min(first_n + row, a.N - 1) * a.ld_ws + (int64_t)(p0 + 4 * c) * 4;
                if (4 * c + 4 <= in_panel) {
                    __builtin_memcpy(&v[x], from, 16);
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e) {
                        uint32_t word = 0;
                        if (4 * c + e < in_panel) __builtin_memcpy(&word, from + 4 * e, 4);
                        v[x][e] = word;
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < C::kPieces; ++x) {
                const int i = threadIdx.x + x * C::kThreads, row = i / pieces, c = i - row * pieces;
                if (row >= 16 * C::kTiles) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (4 * c + e < in_panel) scales[row * stride + 4 * c + e] = v[x][e];
            }
        }
        const uint32_t* words = scales + (16 * NT * nw + r16) * stride + kw;
        const auto fetch = [&](Fp4Operands<MT, NT>& f, int slot) {
            const uint8_t* const from = ring + slot * C::kStage;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                f.w[t] = *reinterpret_cast<const u32x4_t*>(from + w_at + t * 1024);
                f.scale[t] = words[16 * t * stride];
            }
#pragma unroll
            for (int x = 0; x < MT; ++x)
                f.a[x] = operand(*reinterpret_cast<const u32x4_t*>(from + a_at + x * 2048),
                                 *reinterpret_cast<const u32x4_t*>(from + (a_at ^ 64) + x * 2048));
            words += KW;
        };
        const int rounds = NW > 1 ? (in_panel + KW - 1) / KW : count;       // (with a barrier each: the same for all)
        wait_stages<C::kLoads, D - 1>(count - 1);
        __syncthreads();
        Fp4Operands<MT, NT> f[2];
        if (count > 0) fetch(f[0], 0);
        int i = 0, slot = 0;
        // One step: the next one's operands are read, and a stage is loaded where this one's lay, under its products.
        const auto round = [&](auto steady, Fp4Operands<MT, NT>& now, Fp4Operands<MT, NT>& then) {
            constexpr bool kSteady = decltype(steady)::value;
            if constexpr (kSteady) wait_loads<C::kLoads * (D - 2)>();
            else wait_stages<C::kLoads, D - 2>(count - 2 - i);
            __builtin_amdgcn_s_waitcnt(0xc07f);                             // (lgkmcnt(0): this step's operands)
            if constexpr (NW > 1) __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (kSteady || i + D < count) load(slot);
            slot = slot + 1 == D ? 0 : slot + 1;
            if (kSteady || i + 1 < count) fetch(then, slot);
            __builtin_amdgcn_sched_barrier(0);
            if (kSteady || NW == 1 || i < count) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int x = 0; x < MT; ++x) multiply(t, x, now.w[t], now.a[x], now.scale[t] >> (8 * g));
            }
            ++i;
        };
        while (i + D + 1 < count) {
            round(std::true_type(), f[0], f[1]);
            round(std::true_type(), f[1], f[0]);
        }
        while (i < rounds) {
            round(std::false_type(), f[0], f[1]);
            if (i < rounds) round(std::false_type(), f[1], f[0]);
        }
    }
    // The step that K ends in, straight to registers: what lies behind K counts 0.
    if (steps * 128 < K && kw == KW - 1) {
        const int k = steps * 128;
        i32x8_t av[MT];
#pragma unroll
        for (int x = 0; x < MT; ++x) {
            const uint8_t* const row = a.a + min(m0 + 16 * x + r16, a.M - 1) * a.lda;
            u32x4_t lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
            if (k + 16 * g < K) lo = *reinterpret_cast<const u32x4_t*>(row + k + 16 * g);
            if (k + 64 + 16 * g < K) hi = *reinterpret_cast<const u32x4_t*>(row + k + 64 + 16 * g);
            av[x] = operand(lo, hi);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int64_t n = min(n0 + 16 * t + r16, a.N - 1);
            u32x4_t w = {0, 0, 0, 0};
            uint32_t sc = 0;
            if (k + 32 * g < K) {
                w = *reinterpret_cast<const u32x4_t*>(a.w + n * a.ldw + k / 2 + 16 * g);
                sc = a.w_scale[n * a.ld_ws + k / 32 + g];
            }
#pragma unroll
            for (int x = 0; x < MT; ++x) multiply(t, x, w, av[x], sc);
        }
    }

    // ---- a lane holds 4 outputs n of one row m
    const auto store = [&](int t, int x, f32x4_t v) {
        const int64_t m = m0 + 16 * x + r16, col = n0 + 16 * t + 4 * g;
        if (m >= a.M || col >= a.N || (MR == 8 && r16 >= 8)) return;        // (the other 8 are the first again)
        v *= a.a_scale[a.per_tensor ? 0 : m];
        if (a.out_f32) {
            float* const y = reinterpret_cast<float*>(a.y) + m * a.ldy + col;
            if (col + 4 <= a.N) *reinterpret_cast<f32x4_t*>(y) = v;
            else
                for (int e = 0; col + e < a.N; ++e) y[e] = v[e];
        } else {
            uint16_t* const y = reinterpret_cast<uint16_t*>(a.y) + m * a.ldy + col;
            const uint2 o = uint2{f32_to_bf16x2(v[0], v[1]), f32_to_bf16x2(v[2], v[3])};
            if (col + 4 <= a.N) *reinterpret_cast<uint2*>(y) = o;
            else
                for (int e = 0; col + e < a.N; ++e) y[e] = (uint16_t)((e < 2 ? o.x : o.y) >> (16 * (e & 1)));
        }
    };
    if constexpr (KW == 1) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int x = 0; x < MT; ++x) store(t, x, acc[t][x]);
    } else {                                 // the waves' sums, added in their order
        f32x4_t* const box = reinterpret_cast<f32x4_t*>(smem);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int x = 0; x < MT; ++x) box[((kw * NW + nw) * NT * MT + t * MT + x) * 64 + lane] = acc[t][x];
        __syncthreads();
        const f32x4_t* const mine = box + nw * NT * MT * 64 + lane;
        for (int i = kw; i < NT * MT; i += KW) {
            f32x4_t v = mine[i * 64];
#pragma unroll
            for (int j = 1; j < KW; ++j) v += mine[(j * C::kTiles * MT + i) * 64];
            store(i / MT, i % MT, v);
        }
    }
}

template <int MR, int NT, int KW, int NW, int D>
hipError_t launch_fp4_tiles(const Fp4Args& a, hipStream_t stream) {
    using C = Fp4Shape<MR, NT, KW, NW, D>;
    const dim3 grid((unsigned)((a.N + 16 * C::kTiles - 1) / (16 * C::kTiles)), (unsigned)((a.M + MR - 1) / MR));
    hipLaunchKernelGGL((gemm_fp4_kernel<MR, NT, KW, NW, D>), grid, dim3(C::kThreads), C::lds(a.K / 128), stream, a);
    return hipGetLastError();
}

template <size_t... I>
hipError_t launch_fp4_variant(int at, const Fp4Args& a, hipStream_t stream, std::index_sequence<I...>) {
    using Launch = hipError_t (*)(const Fp4Args&, hipStream_t);
    static constexpr Launch launch[] = {launch_fp4_tiles<kFp4Variants[I].mr, kFp4Variants[I].nt, kFp4Variants[I].kw,
                                                         kFp4Variants[I].nw, kFp4Variants[I].d>...};
    return launch[at](a, stream);
}

}  // namespace

hipError_t launch_fp4_quantize(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld_x, uint8_t* q, int64_t ld_q,
                               uint8_t* scales, int64_t ld_s, hipStream_t stream) {
    const dim3 grid((unsigned)((cols / 8 + 255) / 256), (unsigned)(rows < 65535 ? rows : 65535));
    hipLaunchKernelGGL(fp4_quantize_kernel, grid, dim3(256), 0, stream, x, rows, cols, ld_x, q, ld_q, scales, ld_s);
    return hipGetLastError();
}

hipError_t launch_gemm_fp4(const Fp4Args& a, hipStream_t stream) {
    return launch_fp4_variant(plan_fp4(a.M, a.N, a.K), a, stream, std::make_index_sequence<kFp4VariantCount>());
}

}  // namespace specfp8
