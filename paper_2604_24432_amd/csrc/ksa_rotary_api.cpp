// C-ABI entry points of rotary positions.  Every argument check happens before the first HIP call.
#include <cmath>

#include "ksa_paged_checks.h"
#include "ksa_rotary.h"

namespace {

// {batch, row, head} strides of a [B, rows, heads, head_dim] tensor
bool rotary_strides(int64_t out[3], const int64_t *given, int64_t rows, int32_t heads, int32_t head_dim) {
    out[2] = given ? given[2] : head_dim, out[1] = given ? given[1] : (int64_t)heads * head_dim, out[0] = given ? given[0] : rows * heads * head_dim;
    for (int x = 0; x < 3; ++x)
        if (out[x] <= 0 || out[x] % 8 != 0) return false;
    return true;
}

// rows: of a sequence
int rotary_call(const ksa_params *p, const ksa_rotary *rotary, int64_t rows, const void *q, const void *k, void *q_out, void *k_out, const int64_t *qs, const int64_t *ks,
                const int64_t *qos, const int64_t *kos, bool back, const int32_t *pos, int32_t kind, void *stream) {
    if (ksa_check_rotary(rotary, p->head_dim) != KSA_OK) return KSA_ERR_INVALID_ARG;
    if ((q != nullptr) != (q_out != nullptr) || (k != nullptr) != (k_out != nullptr) || (!q && !k)) return KSA_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(q_out, 16) || !aligned(k_out, 16)) return KSA_ERR_INVALID_ARG;
    KsaRotaryCall a;
    const int32_t heads[2] = {p->n_q_heads, p->n_kv_heads};
    const int64_t *const in[2] = {qs, ks}, *const out[2] = {qos, kos};
    a.in[0] = q, a.in[1] = k, a.out[0] = q_out, a.out[1] = k_out;
    for (int x = 0; x < 2; ++x)
        if (!rotary_strides(a.in_strides[x], a.in[x] ? in[x] : nullptr, rows, heads[x], p->head_dim) ||
            !rotary_strides(a.out_strides[x], a.in[x] ? out[x] : nullptr, rows, heads[x], p->head_dim))
            return KSA_ERR_INVALID_ARG;
    if (too_many_waves(rows * p->batch)) return KSA_ERR_UNSUPPORTED;
    a.p = *p, a.rotary = *rotary, a.rows = (int32_t)rows, a.back = back, a.pos = pos, a.kind = kind;
    return ksa_launch_rotary(a, stream);
}
int rotary_call(const ksa_params *p, const ksa_rotary *rotary, const void *q, const void *k, void *q_out, void *k_out, const int64_t *qs, const int64_t *ks,
                const int64_t *qos, const int64_t *kos, bool back, void *stream) {
    const int rc = ksa_validate_params(p);
    return rc != KSA_OK ? rc : rotary_call(p, rotary, augmented(p), q, k, q_out, k_out, qs, ks, qos, kos, back, nullptr, KSA_ROW_TEXT, stream);
}

}  // namespace

extern "C" {

int ksa_rotary_turns(const ksa_rotary_rule *r, uint64_t *turns, float *magnitude) {
    if (!r || !turns || !magnitude || r->dim < 2 || r->dim % 2 != 0 || r->scaling < KSA_ROTARY_PLAIN || r->scaling > KSA_ROTARY_BY_PARTS) return KSA_ERR_INVALID_ARG;
    if (!(r->base > 1.0) || !std::isfinite(r->base)) return KSA_ERR_INVALID_ARG;
    if (r->scaling != KSA_ROTARY_PLAIN && (!(r->factor >= 1.0) || !std::isfinite(r->factor))) return KSA_ERR_INVALID_ARG;
    const bool parts = r->scaling == KSA_ROTARY_BY_PARTS;
    if (parts && (!(r->original > 0.0) || !std::isfinite(r->original) || !(r->slow >= 0.0) || !(r->fast > r->slow) || !std::isfinite(r->fast))) return KSA_ERR_INVALID_ARG;
    const long double turn = 6.283185307179586476925286766559L;
    for (int32_t i = 0; i < r->dim / 2; ++i) {
        long double f = std::pow((long double)r->base, -2.0L * i / r->dim);   // at most 1: less than a sixth of a turn
        if (r->scaling == KSA_ROTARY_LINEAR) f /= r->factor;
        if (parts) {
            long double s = (r->original * f / turn - r->slow) / (r->fast - r->slow);
            s = s < 0 ? 0 : s > 1 ? 1 : s;
            f *= s + (1 - s) / r->factor;
        }
        turns[i] = (uint64_t)std::floor(f / turn * 18446744073709551616.0L + 0.5L);
    }
    *magnitude = parts ? (float)(0.1 * std::log(r->factor) + 1.0) : 1.f;
    return KSA_OK;
}

int ksa_rotary_fwd(const ksa_params *p, const ksa_rotary *rotary, const void *q, const void *k, void *q_out, void *k_out, const int64_t q_strides[3],
                   const int64_t k_strides[3], const int64_t q_out_strides[3], const int64_t k_out_strides[3], void *stream) {
    return rotary_call(p, rotary, q, k, q_out, k_out, q_strides, k_strides, q_out_strides, k_out_strides, false, stream);
}

int ksa_rotary_bwd(const ksa_params *p, const ksa_rotary *rotary, const void *dq_out, const void *dk_out, void *dq, void *dk, const int64_t dq_out_strides[3],
                   const int64_t dk_out_strides[3], const int64_t dq_strides[3], const int64_t dk_strides[3], void *stream) {
    return rotary_call(p, rotary, dq_out, dk_out, dq, dk, dq_out_strides, dk_out_strides, dq_strides, dk_strides, true, stream);
}

int ksa_rotary_step(const ksa_params *p, const ksa_rotary *rotary, int32_t kind, const void *q, const void *k, const int32_t *pos, void *q_out, void *k_out,
                    const int64_t q_strides[2], const int64_t k_strides[2], const int64_t q_out_strides[2], const int64_t k_out_strides[2], void *stream) {
    const int rc = ksa_validate_params(p);
    if (rc != KSA_OK) return rc;
    if ((kind != KSA_ROW_TEXT && kind != KSA_ROW_SUMMARY) || (kind == KSA_ROW_SUMMARY && p->n_summary == 0) || !pos || !aligned(pos, 4)) return KSA_ERR_INVALID_ARG;
    const int64_t *const given[4] = {q_strides, k_strides, q_out_strides, k_out_strides};
    int64_t with_rows[4][3];      // a row's stride is of no account
    for (int x = 0; x < 4; ++x)
        if (given[x]) with_rows[x][0] = with_rows[x][1] = given[x][0], with_rows[x][2] = given[x][1];
    auto strides = [&](int x) { return given[x] ? with_rows[x] : nullptr; };
    return rotary_call(p, rotary, 1, q, k, q_out, k_out, strides(0), strides(1), strides(2), strides(3), false, pos, kind, stream);
}

int ksa_paged_rotary(const ksa_params *p, const ksa_paged_cache *cache, const ksa_rotary *rotary, const void *q, void *q_out, const void *k_new, const void *v_new,
                     const int64_t q_strides[2], const int64_t q_out_strides[2], const int64_t kv_strides[2], const int32_t *cu_rows, const int32_t *start,
                     int64_t total_rows, void *stream) {
    KsaPagedRotary a;
    int rc = move_call(a.move, p, cache, k_new, v_new, kv_strides, cu_rows, start, total_rows);
    if (rc != KSA_OK) return rc;
    if (ksa_check_rotary(rotary, p->head_dim) != KSA_OK) return KSA_ERR_INVALID_ARG;
    if ((q != nullptr) != (q_out != nullptr) || !aligned(q, 16) || !aligned(q_out, 16)) return KSA_ERR_INVALID_ARG;
    if ((rc = check_strides(a.q_strides, q ? q_strides : nullptr, p->n_q_heads, p->head_dim)) != KSA_OK) return rc;
    if ((rc = check_strides(a.out_strides, q ? q_out_strides : nullptr, p->n_q_heads, p->head_dim)) != KSA_OK) return rc;
    if (too_many_waves(total_rows)) return KSA_ERR_UNSUPPORTED;
    if (total_rows == 0) return KSA_OK;
    a.move.k = const_cast<void *>(k_new), a.move.v = const_cast<void *>(v_new);   // (read only)
    a.rotary = *rotary, a.q = q, a.q_out = q_out;
    return ksa_launch_paged_rotary(a, stream);
}

}  // extern "C"
