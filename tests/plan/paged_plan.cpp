// Prints what ksa_paged_fwd launches, for each line of standard input (batch, heads, KV heads, head_dim, tokens, chunk length, summaries, window
// chunks, new rows, most of a sequence, spans (0: the library's choice), bytes of workspace (-1: what the library asks for)): status, whether it
// is the kernel for few rows, spans, pairs of a query tile, groups of waves, query tiles, and the bytes that the library asks for.  Launches end here:
// nothing reaches a GPU.
#include <cstdio>

#include "ksa.h"
#include "ksa_paged.h"

static KsaPagedPlan seen;

int ksa_launch_paged_append(const KsaPagedMove &, void *) { return KSA_ERR_HIP; }
int ksa_launch_paged_read(const KsaPagedMove &, void *) { return KSA_ERR_HIP; }
int ksa_launch_paged_fwd(const KsaPagedFwd &L, void *) {
    seen = L.plan;
    return KSA_OK;
}

int main() {
    int B, Hq, Hkv, d, n, c, m, C, n_splits;
    long long total, most, given;
    while (std::scanf("%d %d %d %d %d %d %d %d %lld %lld %d %lld", &B, &Hq, &Hkv, &d, &n, &c, &m, &C, &total, &most, &n_splits, &given) == 12) {
        ksa_params p{};
        p.batch = B, p.n_q_heads = Hq, p.n_kv_heads = Hkv, p.head_dim = d, p.n_text = n, p.chunk_len = c, p.n_summary = m, p.window_chunks = C;
        p.compress_ratio = m ? c / m : 0;
        alignas(16) static char x[16];   // (never read)
        ksa_paged_cache cache{};
        cache.page_rows = 16, cache.n_pages = cache.text_pages = cache.summary_pages = 1;
        cache.text_table = cache.summary_table = (const int32_t *)x, cache.k = cache.v = x;
        seen = KsaPagedPlan{};
        const size_t asked = ksa_paged_workspace_bytes(&p, total, most, n_splits), bytes = given < 0 ? asked : (size_t)given;
        const int rc = ksa_paged_fwd(&p, &cache, x, x, nullptr, nullptr, nullptr, (const int32_t *)x, (const int32_t *)x, total, most,
                                     bytes > 0 ? x : nullptr, bytes, n_splits, nullptr);
        std::printf("%d %d %d %d %d %d %zu\n", rc, (int)seen.few, seen.n_splits, seen.pairs, seen.groups, seen.slots, asked);
    }
    return 0;
}
