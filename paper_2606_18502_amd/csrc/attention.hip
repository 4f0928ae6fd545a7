// Tree attention masks, and the launches of the attentions: over the paged FP8 cache
// (attn_stream.hpp for few rows, attn_tile.hpp for many, the kernel below for heads
// whose codes are no whole 16-byte pieces) and over packed prompts (attn_tile.hpp).
#include <algorithm>

#include "attn_common.hpp"
#include "attn_stream.hpp"
#include "attn_tile.hpp"

namespace specfp8 {

namespace {

// ---- tree masks: for token-tree verification, for every node of a
// drafted tree, the set of tree nodes its row may attend to (the nodes on the
// path from the root to it, itself included) as a 64-bit mask, and its depth.
//
// One wave per sequence, lane n owning node n (N <= 64).  The masks come from
// pointer jumping over the parent links: after step s every lane holds the
// nodes within 2^s - 1 steps above it and a pointer to its 2^s-th ancestor,
// so six steps of lane exchanges (no memory traffic) cover any depth up to
// 64.  A node whose parent is not one of the earlier nodes (or -1) poisons
// itself and, through the same exchanges, every node below it.
constexpr int kTmThreads = 256;
constexpr int kTmSeqPerBlock = kTmThreads / 64;

__global__ __launch_bounds__(kTmThreads) void tree_mask_kernel(const int32_t* __restrict__ parents, int64_t B,
                                                               int N, uint64_t* __restrict__ mask,
                                                               int32_t* __restrict__ depth) {
    const int lane = threadIdx.x & 63;
    const int64_t b = (int64_t)blockIdx.x * kTmSeqPerBlock + threadIdx.x / 64;   // wave-uniform
    if (b >= B) return;
    const bool node = lane < N;
    const int p = node ? parents[b * N + lane] : -1;
    int bad = (node && (p < -1 || p >= lane)) ? 1 : 0;
    uint32_t lo = 0, hi = 0;                  // the mask, as two halves for the lane exchanges
    if (node) {
        if (lane < 32) lo = 1u << lane;
        else hi = 1u << (lane - 32);
    }
    int anc = bad ? -1 : p;
#pragma unroll
    for (int s = 0; s < 6; ++s) {
        const int src = anc >= 0 ? anc : lane;
        const uint32_t lo_up = __shfl(lo, src);
        const uint32_t hi_up = __shfl(hi, src);
        const int bad_up = __shfl(bad, src);
        const int anc_up = __shfl(anc, src);
        if (anc >= 0) {
            lo |= lo_up;
            hi |= hi_up;
            bad |= bad_up;
            anc = anc_up;
        }
    }
    if (!node) return;
    const uint64_t m = bad ? 0ull : (((uint64_t)hi << 32) | lo);
    mask[b * N + lane] = m;
    depth[b * N + lane] = bad ? 0 : __popcll(m);
}


// ---- attention ----------------------------------------------------------------
constexpr int kRowThreads = 256, kRowWaves = kRowThreads / kWave, kMaxD = 256;

// Which sequence row t belongs to: the last b with cu[b] <= t (-1: none).
__device__ __forceinline__ int seq_of(const int32_t* cu, int T, int B, int t) {
    if (!cu) return t / (T / B);
    int lo = 0, hi = B;                       // cu[lo] <= t < cu[hi], if anywhere
    if (t < cu[0] || t >= cu[B]) return -1;
    while (hi - lo > 1) {
        const int m = (lo + hi) / 2;
        if (cu[m] <= t) lo = m;
        else hi = m;
    }
    return lo;
}

// Heads whose rows are not whole 16-byte pieces of codes (D % 16 == 8): one wave per (row, query head),
// lanes over 64 keys for the scores, then over D for the sums.  All fp32 on the vector units, 64 keys a step,
// the running maximum and sum of the softmax; bounded by its dot products (every wave reads its keys again).
__device__ __forceinline__ void attend_row(const PagedArgs& a, const float* qs, int b, int t, int head) {
    const int lane = threadIdx.x % kWave, D = a.D, H = a.H, kvh = head / (a.Hq / H);
    int first, n;
    rows_of(a.cu_q, a.T, a.B, b, &first, &n);
    const int L = min(max(a.kv_lens[b], 0), a.max_len), i = t - first, last = a.tree ? L - 1 : L - n + i;
    const uint64_t mask = a.tree && i > 0 ? a.tree[(int64_t)b * a.N + i - 1] : 0;
    float m = -INFINITY, sum = 0.0f, o[kMaxD / kWave] = {};
    for (int j0 = 0; j0 <= last; j0 += kWave) {
        const int j = j0 + lane;
        bool seen = j <= last;
        if (a.tree && seen && j >= L - a.N) seen = (mask >> (j - (L - a.N))) & 1;
        int page = -1;
        if (seen) page = a.tables[(int64_t)b * a.ld_tables + j / a.block_size];
        seen = seen && page >= 0 && page < a.num_blocks;
        const int64_t at = seen ? ((int64_t)page * a.block_size + j % a.block_size) * H + kvh : 0;
        float s = -INFINITY, sv = 1.0f;
        if (seen) {
            s = 0.0f;
            for (int d = 0; d < D; d += 8) {
                const uint2 c = *reinterpret_cast<const uint2*>(a.k_cache + at * D + d);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t x = (e < 4 ? c.x : c.y) >> (8 * (e & 3));
                    s = fmaf(qs[d + e], __builtin_amdgcn_cvt_f32_fp8((int)x, 0), s);
                }
            }
            s *= (a.per_tensor ? a.k_scale[0] : a.k_scale[at]) * (a.scale * 1.44269504f);
            sv = a.per_tensor ? a.v_scale[0] : a.v_scale[at];
        }
        const float top = fmaxf(m, wave_max(s));
        const float ref = top == -INFINITY ? 0.0f : top;
        const float down = exp2f(m - ref), p = exp2f(s - ref);
        sum = sum * down + wave_sum(p);
#pragma unroll
        for (int x = 0; x < kMaxD / kWave; ++x) o[x] *= down;
        m = top;
        const uint64_t any = __ballot(seen);
        const float pv = p * sv;
        for (int u = 0; u < kWave; ++u) {
            if (!((any >> u) & 1)) continue;
            const float pu = __shfl(pv, u);
            const int64_t au = __shfl(at, u);
#pragma unroll
            for (int x = 0; x < kMaxD / kWave; ++x) {
                const int d = lane + kWave * x;
                if (d < D) o[x] = fmaf(pu, __builtin_amdgcn_cvt_f32_fp8(a.v_cache[au * D + d], 0), o[x]);
            }
        }
    }
    uint16_t* out = a.out + (int64_t)t * a.ld_out + (int64_t)head * D;
#pragma unroll
    for (int x = 0; x < kMaxD / kWave; ++x) {
        const int d = lane + kWave * x;
        if (d < D) out[d] = (uint16_t)f32_to_bf16x2(sum != 0.0f ? o[x] / sum : 0.0f, 0.0f);
    }
}

__global__ __launch_bounds__(kRowThreads) void attention_row_kernel(PagedArgs a) {
    __shared__ float qs[kRowWaves][kMaxD];
    const int w = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int64_t items = (int64_t)a.T * a.Hq;
    for (int64_t at = (int64_t)blockIdx.x * kRowWaves; at < items; at += (int64_t)gridDim.x * kRowWaves) {
        const int64_t item = at + w;
        const int t = (int)(item / a.Hq), head = (int)(item % a.Hq);
        const int b = item < items ? seq_of(a.cu_q, a.T, a.B, t) : -1;
        __syncthreads();                      // the last item's reads
        if (b >= 0)
            for (int d = lane; d < a.D; d += kWave) qs[w][d] = bf16_to_f32(a.q[(int64_t)t * a.ld_q + (int64_t)head * a.D + d]);
        __syncthreads();
        if (b >= 0) attend_row(a, qs[w], b, t, head);
    }
}

// The lengths are the device's: never more workgroups than there are cells where every sequence fills its table.
int workgroups(const PagedPlan& p, int64_t units, int64_t cells) {
    return (int)std::min<int64_t>(std::min<int64_t>(units, p.groups) * cells, p.groups);
}

template <int DP, int NQ, int HG>
hipError_t launch_stream(const PagedPlan& p, const PagedArgs& a, void* workspace, hipStream_t stream) {
    using C = StreamShape<DP, NQ, HG>;
    const int64_t units = ((int64_t)a.T * (a.Hq / a.H) / C::kRows + a.B) * ((a.H + HG - 1) / HG);
    const int grid = workgroups(p, units, std::max<int64_t>(((a.max_len + C::kStep - 1) / C::kStep + 1) / kStreamCell, 1));
    float* const part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(workspace) + kAttnTicketBytes);
    hipLaunchKernelGGL((paged_stream_kernel<DP, NQ, HG>), dim3(grid), dim3(64 * kStreamWaves), C::kLds, stream, a, part,
                       reinterpret_cast<unsigned int*>(workspace), grid, C::KW == 1 ? 5 : 3);
    return hipGetLastError();
}

template <int DP>
hipError_t launch_tiles(const PagedPlan& p, const PagedArgs& a, void* workspace, hipStream_t stream) {
    constexpr int kRows = 32 * kTileWaves<DP>, kKeys = TileShape_<DP>::kKeys;
    constexpr int kLds = std::max(PagedTileShape<DP>::kLds, kRows * DP * 4);
    const int64_t units = ((int64_t)a.T * (a.Hq / a.H) / kRows + a.B) * a.H;
    const int grid = workgroups(p, units, std::max<int64_t>(((a.max_len + kKeys - 1) / kKeys + 1) / kTileCell, 1));
    float* const part = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(workspace) + kAttnTicketBytes);
    unsigned int* const tickets = reinterpret_cast<unsigned int*>(workspace);
    const dim3 block(64 * kTileWaves<DP>);
    if (a.per_tensor)
        hipLaunchKernelGGL((paged_tile_kernel<DP, true>), dim3(grid), block, kLds, stream, a, part, tickets, grid, 3);
    else
        hipLaunchKernelGGL((paged_tile_kernel<DP, false>), dim3(grid), block, kLds, stream, a, part, tickets, grid, 3);
    return hipGetLastError();
}

template <int DP>
hipError_t launch_paged(const PagedPlan& p, const PagedArgs& a, void* workspace, hipStream_t stream) {
    if (p.tiles) return launch_tiles<DP>(p, a, workspace, stream);
    if (p.hg == 1)
        return p.nq == 1 ? launch_stream<DP, 1, 1>(p, a, workspace, stream) : launch_stream<DP, 2, 1>(p, a, workspace, stream);
    if (p.hg == 2)
        return p.nq == 1 ? launch_stream<DP, 1, 2>(p, a, workspace, stream) : launch_stream<DP, 2, 2>(p, a, workspace, stream);
    return launch_stream<DP, 1, 4>(p, a, workspace, stream);
}

}  // namespace

hipError_t launch_paged_attention(const PagedArgs& given, void* workspace, hipStream_t stream) {
    PagedArgs a = given;
    if (a.num_blocks == 0) {             // no cache: every page is outside it, and loads need some address (q's first row)
        a.k_cache = a.v_cache = reinterpret_cast<const uint8_t*>(a.q);
        a.k_scale = a.v_scale = reinterpret_cast<const float*>(a.q);
        a.per_tensor = 0;                // (a scale of a whole tensor would reach the sums)
    }
    const PagedPlan p = plan_paged(a.T, a.B, a.Hq, a.H, a.D, a.max_len);
    if (p.dp == 64) return launch_paged<64>(p, a, workspace, stream);
    if (p.dp == 128) return launch_paged<128>(p, a, workspace, stream);
    if (p.dp == 256) return launch_paged<256>(p, a, workspace, stream);
    const int64_t blocks = std::min<int64_t>(((int64_t)a.T * a.Hq + kRowWaves - 1) / kRowWaves, (1 << 24) - 1);
    hipLaunchKernelGGL(attention_row_kernel, dim3((unsigned)blocks), dim3(kRowThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_prompt_attention(const PromptArgs& a, hipStream_t stream) {
    const int64_t slots = prompt_slots(a.T, a.B, a.Hq, a.H);
    const dim3 grid((unsigned)(slots * a.H)), block(256);
    if (a.D > 128)
        hipLaunchKernelGGL(prompt_tile_kernel<256>, grid, block, TileShape_<256>::kLds, stream, a, (int)slots);
    else if (a.D <= 64)
        hipLaunchKernelGGL(prompt_tile_kernel<64>, grid, block, TileShape_<64>::kLds, stream, a, (int)slots);
    else
        hipLaunchKernelGGL(prompt_tile_kernel<128>, grid, block, TileShape_<128>::kLds, stream, a, (int)slots);
    return hipGetLastError();
}

hipError_t launch_tree_mask(const int32_t* parents, int64_t B, int64_t N, uint64_t* mask, int32_t* depth,
                            hipStream_t stream) {
    const int64_t blocks = (B + kTmSeqPerBlock - 1) / kTmSeqPerBlock;
    hipLaunchKernelGGL(tree_mask_kernel, dim3((unsigned)blocks), dim3(kTmThreads), 0, stream, parents, B, (int)N,
                       mask, depth);
    return hipGetLastError();
}

}  // namespace specfp8
