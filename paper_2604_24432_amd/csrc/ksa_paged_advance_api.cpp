// C-ABI entry points of a step's rows and pages.  Every argument check happens before the first HIP call.
#include "ksa_paged_checks.h"

namespace {

// Columns for which every index and count of them fits 32 bits, a workgroup's step behind the last one among them.
constexpr int64_t MOST_COLUMNS = ((int64_t)1 << 31) - 4096;
bool too_large(const ksa_params *p, const ksa_paged_cache *cache) {
    return p->batch * ((int64_t)cache->text_pages + cache->summary_pages) >= MOST_COLUMNS;
}

size_t bytes_of(const ksa_params *p, const ksa_paged_cache *cache) { return (ksa_paged_advance_ints(p->batch, cache->n_pages) * sizeof(int32_t) + 15) / 16 * 16; }

}  // namespace

extern "C" {

size_t ksa_paged_advance_workspace_bytes(const ksa_params *p, const ksa_paged_cache *cache) {
    KsaPagedCall call;
    if (ksa_validate_params(p) != KSA_OK || check_cache(call, p, cache) != KSA_OK || too_large(p, cache)) return 0;
    return bytes_of(p, cache);
}

int ksa_paged_advance(const ksa_params *p, const ksa_paged_cache *cache, int32_t *page_refs, const int32_t *held, const int32_t *new_text, int32_t *cu_rows, int32_t *start,
                      int32_t *lacking, int64_t *slots, int32_t *positions, int32_t *tokens, int64_t total_rows, void *workspace, size_t workspace_bytes, void *stream) {
    KsaPagedAdvance a;
    int rc = ksa_validate_params(p);
    if (rc != KSA_OK) return rc;
    if ((rc = check_cache(a.call, p, cache)) != KSA_OK) return rc;
    if (!page_refs || !held || !new_text || !cu_rows || !start || !lacking || total_rows < 0) return KSA_ERR_INVALID_ARG;
    for (const void *x : {static_cast<const void *>(page_refs), static_cast<const void *>(held), static_cast<const void *>(new_text), static_cast<const void *>(cu_rows),
                          static_cast<const void *>(start), static_cast<const void *>(lacking), static_cast<const void *>(positions), static_cast<const void *>(tokens)})
        if (!aligned(x, 4)) return KSA_ERR_INVALID_ARG;
    if (!aligned(slots, 8) || !aligned(workspace, 16)) return KSA_ERR_INVALID_ARG;
    if (too_large(p, cache) || total_rows >= ((int64_t)1 << 31) - 256) return KSA_ERR_UNSUPPORTED;
    const size_t need = bytes_of(p, cache);
    if (!workspace) return KSA_ERR_INVALID_ARG;
    if (workspace_bytes < need) return KSA_ERR_WORKSPACE_TOO_SMALL;
    a.call.cu_rows = cu_rows, a.call.start = start, a.call.total_rows = (int32_t)total_rows;
    a.page_refs = page_refs, a.held = held, a.new_text = new_text, a.cu_rows = cu_rows, a.start = start, a.lacking = lacking;
    a.slots = slots, a.positions = positions, a.tokens = tokens, a.workspace = static_cast<int32_t *>(workspace);
    return ksa_launch_paged_advance(a, stream);
}

}  // extern "C"
