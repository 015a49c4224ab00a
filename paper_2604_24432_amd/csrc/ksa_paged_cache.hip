// Rows into and out of a paged cache of bf16 or 8-bit rows.
#include "ksa_paged_move.h"

#define KSA_LAUNCH_MOVE(KERNEL)                                                                                                        \
    const MoveArgs a = move_args(L);                                                                                                  \
    const int d = L.call.p.head_dim;                                                                                                  \
    const bool f8 = L.call.cache.format == KSA_CACHE_FP8;                                                                             \
    const dim3 grid = move_grid(a, d);                                                                                                \
    hipStream_t st = static_cast<hipStream_t>(stream);                                                                                \
    if (d == 128 && f8) hipLaunchKernelGGL((KERNEL<128, KSA_CACHE_FP8>), grid, dim3(256), 0, st, a);                                  \
    else if (d == 128) hipLaunchKernelGGL((KERNEL<128, KSA_CACHE_BF16>), grid, dim3(256), 0, st, a);                                  \
    else if (f8) hipLaunchKernelGGL((KERNEL<64, KSA_CACHE_FP8>), grid, dim3(256), 0, st, a);                                          \
    else hipLaunchKernelGGL((KERNEL<64, KSA_CACHE_BF16>), grid, dim3(256), 0, st, a);                                                 \
    return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP

int ksa_launch_paged_append(const KsaPagedMove &L, void *stream) {
    if (L.call.cache.format == KSA_CACHE_FP4) {
        ksa_launch_paged_append_fp4(L, stream);
        return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP;
    }
    KSA_LAUNCH_MOVE(ksa_paged_append_kernel);
}
int ksa_launch_paged_read(const KsaPagedMove &L, void *stream) {
    if (L.call.cache.format == KSA_CACHE_FP4) {
        ksa_launch_paged_read_fp4(L, stream);
        return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP;
    }
    KSA_LAUNCH_MOVE(ksa_paged_read_kernel);
}
