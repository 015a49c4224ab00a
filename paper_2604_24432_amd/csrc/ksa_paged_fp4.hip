// Attention over a paged cache of 4-bit rows.
#include "ksa_paged_fwd.h"

namespace {

template <int D>
void launch(const FwdArgs &a, const KsaPagedPlan &plan, hipStream_t st) {
    if (plan.few) launch_few<D, KSA_CACHE_FP4>(a, plan, st);
    else launch_many<D, KSA_CACHE_FP4>(a, plan, st);
}

}  // namespace

void ksa_launch_paged_fwd_fp4(const KsaPagedFwd &L, void *stream) {
    const FwdArgs a = fwd_args(L);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (L.call.p.head_dim == 128) launch<128>(a, L.plan, st);
    else launch<64>(a, L.plan, st);
}
