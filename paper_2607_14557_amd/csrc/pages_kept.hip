// The plan of a step in a cache whose tokens an eviction may have cut (page_plan.h).
#include "page_plan.h"

namespace seer {

int launch_page_plan_kept(const PagePlanParams& p, const int* kept, hipStream_t s) { return launch_plan(KeptParams{p, kept}, s); }

}  // namespace seer
