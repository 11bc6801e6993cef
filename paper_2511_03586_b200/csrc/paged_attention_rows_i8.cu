// The row kernels of the attention over an int8 cache.
#include "paged_rows_q8.cuh"

namespace pd {
namespace paged {

pd_status launch_rows_i8(const pd_paged_attention_desc& d, const Params& p, const Plan& plan, const Scales& scales, const void* k_cache,
                         const void* v_cache, cudaStream_t s) {
  return d.head_dim == 64 ? launch_plan<PD_I8, 64>(d, p, plan, scales, k_cache, v_cache, s) : launch_plan<PD_I8, 128>(d, p, plan, scales, k_cache, v_cache, s);
}

}  // namespace paged
}  // namespace pd
