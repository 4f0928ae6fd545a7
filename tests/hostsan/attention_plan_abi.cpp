// Test-only C view of the paged attention's plan (plan.cpp), so that host
// tests can tell which kernel a call runs.
#include "../../paper_2606_18502_amd/csrc/kernels.hpp"
#include "../../paper_2606_18502_amd/csrc/plan.hpp"

extern "C" {

// out: D padded (0: the row kernel), 16s of rows, KV heads a workgroup, tiles or stream, workgroups at most, workspace
void test_plan_paged(int64_t T, int64_t B, int64_t Hq, int64_t H, int64_t D, int64_t max_len, int64_t* out) {
    const specfp8::PagedPlan p = specfp8::plan_paged(T, B, Hq, H, D, max_len);
    out[0] = p.dp;
    out[1] = p.nq;
    out[2] = p.hg;
    out[3] = p.tiles;
    out[4] = p.groups;
    out[5] = (int64_t)p.bytes;
}

}  // extern "C"
