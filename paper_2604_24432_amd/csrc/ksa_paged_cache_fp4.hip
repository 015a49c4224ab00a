// Rows into and out of a paged cache of 4-bit rows.
#include "ksa_paged_move.h"

void ksa_launch_paged_append_fp4(const KsaPagedMove &L, void *stream) {
    const MoveArgs a = move_args(L);
    const int d = L.call.p.head_dim;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d == 128) hipLaunchKernelGGL((ksa_paged_append_kernel<128, KSA_CACHE_FP4>), move_grid(a, d), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((ksa_paged_append_kernel<64, KSA_CACHE_FP4>), move_grid(a, d), dim3(256), 0, st, a);
}

void ksa_launch_paged_read_fp4(const KsaPagedMove &L, void *stream) {
    const MoveArgs a = move_args(L);
    const int d = L.call.p.head_dim;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d == 128) hipLaunchKernelGGL((ksa_paged_read_kernel<128, KSA_CACHE_FP4>), move_grid(a, d), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((ksa_paged_read_kernel<64, KSA_CACHE_FP4>), move_grid(a, d), dim3(256), 0, st, a);
}
