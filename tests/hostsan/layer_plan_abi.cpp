// Test-only C view of the plans of the rotation into the cache and of 4-bit
// linears (plan.hpp, plan.cpp), so that host tests can tell what a call runs.
#include "../../paper_2606_18502_amd/csrc/plan.hpp"

extern "C" {

int test_rope_log_parts(int64_t T, int64_t Hq, int64_t H, int g) { return specfp8::rope_log_parts(T, Hq, H, g); }
int64_t test_rope_step() { return specfp8::kRopeStep; }

// out: the variant's five numbers, and the steps of a panel of its scales
void test_plan_fp4(int64_t M, int64_t N, int64_t K, int* out) {
    const specfp8::Fp4Variant v = specfp8::kFp4Variants[specfp8::plan_fp4(M, N, K)];
    out[0] = v.mr;
    out[1] = v.nt;
    out[2] = v.kw;
    out[3] = v.nw;
    out[4] = v.d;
    out[5] = specfp8::fp4_panel(v.nt * v.nw);
}
int test_fp4_variants() { return specfp8::kFp4VariantCount; }

}  // extern "C"
