// Test-only C view of the plans of the rotation into the cache (plan.hpp), so
// that host tests can tell what a call runs.
#include "../../paper_2606_18502_amd/csrc/plan.hpp"

extern "C" {

int test_rope_log_parts(int64_t T, int64_t Hq, int64_t H, int g) { return specfp8::rope_log_parts(T, Hq, H, g); }
int64_t test_rope_step() { return specfp8::kRopeStep; }

}  // extern "C"
