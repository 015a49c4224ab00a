// Attention over a paged cache of bf16 or 8-bit rows, and the join of spans' records for all formats.
#include "ksa_paged_fwd.h"

namespace {

// ---- the spans' records joined by log-sum-exp -------------------------------------------------------------------------------

// Bound by the records' bytes and, for few of them, by three loads one behind the other.  At most MOST spans: D / 4 lanes per (row, query head), every
// span's record (the last one's again for those behind it) on its way before the row's sequence is looked up: 20480 items of two spans 7.0 us (a wave for
// each 11.7; 8 records loaded by branches 18), 128 items 4.1.
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <int D, int MOST>
__global__ __launch_bounds__(256) void ksa_paged_join_few_kernel(const FwdArgs a) {
    constexpr int LANES = D / 4, REC = D + 4;
    const int n_items = a.rows.total * a.n_q_heads, first = (int)(blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * (64 / LANES);
    if (first >= n_items) return;
    const int own = first + (int)(threadIdx.x & 63) / LANES, item = min(own, n_items - 1), piece = threadIdx.x % LANES;
    const int n = a.n_splits;
    const float *const rec = a.ws + (int64_t)item * n * REC;
    f32x4 o[MOST];
    f32x2 of[MOST];   // maximum and sum
#pragma unroll
    for (int s = 0; s < MOST; ++s) {
        const float *const at = rec + min(s, n - 1) * REC;
        o[s] = *reinterpret_cast<const f32x4 *>(at + piece * 4), of[s] = *reinterpret_cast<const f32x2 *>(at + D);
    }
    const int row = ksa_div(item, a.by_q_heads), hq = item - row * a.n_q_heads;
    int b;
    const NewRows seq = sequence_of<64 / LANES>(a.rows, ksa_div(first, a.by_q_heads), row, a.max_rows, b);
    if (own >= n_items || row < seq.first || row >= seq.first + seq.n) return;
    float M = LOWEST, den = 0.f;
    f32x4 out = {0.f, 0.f, 0.f, 0.f};
    if (seq.ok) {
#pragma unroll
        for (int s = 0; s < MOST; ++s) M = fmaxf(M, of[s][0]);
#pragma unroll
        for (int s = 0; s < MOST; ++s) {
            const float w = s < n ? __builtin_amdgcn_exp2f(of[s][0] - M) : 0.f;
            den += of[s][1] * w, out += o[s] * w;
        }
    } else den = __builtin_nanf("");
    bf16x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = (__bf16)(out[e] / den);
    *reinterpret_cast<bf16x4 *>(a.o + row * a.o_row + hq * a.o_head + piece * 4) = r;
    if (a.lse && piece == 0) a.lse[item] = log_sum(M, den);
}

// More spans: a workgroup per (row, query head), its four waves each with every fourth group of 8 spans, whose loads travel together; the
// weights of 64 spans live in the lanes of every wave.
template <int D>
__global__ __launch_bounds__(256) void ksa_paged_join_kernel(const FwdArgs a) {
    constexpr int EACH = D / 64, REC = D + 4, MU = 8, PARTS = 4;
    typedef float each __attribute__((ext_vector_type(EACH)));
    const int lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = blockIdx.x;   // row * n_q_heads + query head
    const int n = a.n_splits;
    const float *const rec = a.ws + (int64_t)item * n * REC;
    auto at = [&](int s) { return rec + (int64_t)min(s, n - 1) * REC; };
    f32x2 of = *reinterpret_cast<const f32x2 *>(at(lane) + D);   // maximum and sum
    const int row = ksa_div(item, a.by_q_heads), hq = item - row * a.n_q_heads;
    int b;
    const NewRows seq = sequence_of<1>(a.rows, row, row, a.max_rows, b);
    const bool any = row >= seq.first && row < seq.first + seq.n;
    each out;
#pragma unroll
    for (int e = 0; e < EACH; ++e) out[e] = 0.f;
    float M = LOWEST, den = 0.f;
    if (any && seq.ok) {
        M = of[0];
        for (int s = 64; s < n; s += 64) M = fmaxf(M, at(s + lane)[D]);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
        for (int s = 0; s < n; s += 64) {
            if (s > 0) of = *reinterpret_cast<const f32x2 *>(at(s + lane) + D);
            const float w = __builtin_amdgcn_exp2f(of[0] - M);
            den += s + lane < n ? of[1] * w : 0.f;
            for (int x = MU * part; x < min(64, n - s); x += MU * PARTS) {
                each o[MU];
#pragma unroll
                for (int u = 0; u < MU; ++u) o[u] = *reinterpret_cast<const each *>(at(s + x + u) + lane * EACH);
#pragma unroll
                for (int u = 0; u < MU; ++u)
                    if (s + x + u < n) out += o[u] * __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), x + u));
            }
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) den += __shfl_xor(den, d);
    }
    __shared__ each parts[PARTS][64];
    parts[part][lane] = out;
    __syncthreads();
    if (part > 0 || !any) return;
#pragma unroll
    for (int y = 1; y < PARTS; ++y) out += parts[y][lane];
    if (!seq.ok) den = __builtin_nanf("");
    typedef __bf16 each_bf16 __attribute__((ext_vector_type(EACH)));
    each_bf16 r;
#pragma unroll
    for (int e = 0; e < EACH; ++e) r[e] = (__bf16)(out[e] / den);
    *reinterpret_cast<each_bf16 *>(a.o + row * a.o_row + hq * a.o_head + lane * EACH) = r;
    if (a.lse && lane == 0) a.lse[item] = log_sum(M, den);
}

template <int D>
void launch_join(const FwdArgs &a, hipStream_t st) {
    const int items = a.rows.total * a.n_q_heads;
    const dim3 join((items + 1024 / D - 1) / (1024 / D));
    if (a.n_splits > 8) hipLaunchKernelGGL((ksa_paged_join_kernel<D>), dim3(items), dim3(256), 0, st, a);
    else if (a.n_splits > 4) hipLaunchKernelGGL((ksa_paged_join_few_kernel<D, 8>), join, dim3(256), 0, st, a);
    else if (a.n_splits > 2) hipLaunchKernelGGL((ksa_paged_join_few_kernel<D, 4>), join, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((ksa_paged_join_few_kernel<D, 2>), join, dim3(256), 0, st, a);
}

template <int D, int F>
void launch(const FwdArgs &a, const KsaPagedPlan &plan, hipStream_t st) {
    if (plan.few) launch_few<D, F>(a, plan, st);
    else launch_many<D, F>(a, plan, st);
}

}  // namespace

int ksa_launch_paged_fwd(const KsaPagedFwd &L, void *stream) {
    const FwdArgs a = fwd_args(L);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int d = L.call.p.head_dim, format = L.call.cache.format;
    if (format == KSA_CACHE_FP4) ksa_launch_paged_fwd_fp4(L, stream);
    else if (d == 128) format == KSA_CACHE_FP8 ? launch<128, KSA_CACHE_FP8>(a, L.plan, st) : launch<128, KSA_CACHE_BF16>(a, L.plan, st);
    else format == KSA_CACHE_FP8 ? launch<64, KSA_CACHE_FP8>(a, L.plan, st) : launch<64, KSA_CACHE_BF16>(a, L.plan, st);
    if (L.plan.n_splits > 1) d == 128 ? launch_join<128>(a, st) : launch_join<64>(a, st);
    return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP;
}
