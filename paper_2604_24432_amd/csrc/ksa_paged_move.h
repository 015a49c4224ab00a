// Rows into and out of the paged cache, as bf16, as e4m3 numbers with one power of two per row and KV head, or as e2m1 numbers with one per 32 of them.  Data movement, bound by
// HBM: 16 bytes of a row per lane, the row's largest magnitude by lane moves, the table looked up by every row's lanes.  36864 rows, 8 heads,
// d 128, 8-bit: in 56 us and out again 34, 454 MB at 5.0 TB/s (a copy on this card 5.0); 54000 rows, 16 heads, bf16, out 100 us, 5.3 TB/s; the 36864 rows in 4 bits
// in 43 us, 4.5 TB/s, and out again 30; 64 rows
// of 64 sequences 2.8 us, a launch and three loads one behind the other.  Loads of the new rows in front of the lookup (in 61 / 3.3 us),
// two or four rows per lane (66 / 3.9, 69 / 5.0) did not pay.
#ifndef KSA_PAGED_MOVE_H_
#define KSA_PAGED_MOVE_H_

#include <hip/hip_runtime.h>

#include "ksa_paged.h"

namespace {

struct MoveArgs {
    PagedRows rows;
    __bf16 *k, *v;                // [total_rows, Hkv, d]
    int64_t row_stride, head_stride;
    unsigned char *kc, *vc;       // the pool
    uint8_t *k_exp, *v_exp;
    int64_t page_bytes, head_bytes, row_bytes;
    int32_t n_kv_heads;
    KsaDivisor by_heads;
};

// A block takes 2048 / D neighbouring packed rows of one KV head, which mostly lie side by side in a page, 8 elements per lane; heads fastest.
// (Against a block of 16 neighbouring (row, head) pairs: 54000 rows out 104 us -> 100, 36864 rows out 36 -> 34.)
struct Place {
    int row, head, page, slot;
    bool any;                     // the row is a sequence's
};
template <int LANES>
__device__ __forceinline__ Place place_of(const MoveArgs &a, int group, int head) {
    constexpr int ROWS = 256 / LANES;
    const int first = group * ROWS + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (64 / LANES), row = first + (threadIdx.x & 63) / LANES;
    Place p = {row, head, -1, 0, false};
    if (first >= a.rows.total) return p;
    int b;
    const NewRows r = sequence_of<64 / LANES>(a.rows, first, row, a.rows.total, b);
    p.any = p.row >= r.first && p.row < r.first + r.n;
    if (!p.any || !r.ok) return p;
    const Spot s = spot_of(a.rows, entry_of(a.rows, b, kind_of(a.rows, r.start + (p.row - r.first))));
    p.page = s.page, p.slot = s.slot;
    return p;
}

template <int CTRL>
__device__ __forceinline__ unsigned dpp_umax(unsigned x) {
    return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false));
}

// The biased exponent of a row's power of two, from the lane's 8 elements, in all lanes of the row.
template <int LANES>
__device__ __forceinline__ int row_exponent(const u32x4 &x) {
    unsigned most = 0;   // largest finite magnitude, as the bits of a bf16
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned lo = x[e] & 0x7fffu, hi = (x[e] >> 16) & 0x7fffu;
        most = max(most, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
    }
    most = dpp_umax<0xB1>(most);    // quad_perm [1,0,3,2]
    most = dpp_umax<0x4E>(most);    // quad_perm [2,3,0,1]
    most = dpp_umax<0x141>(most);   // row_half_mirror
    if (LANES == 16) most = dpp_umax<0x140>(most);   // row_mirror
    // most = 1.f * 2^(E - 127), and 448 = 1.75 * 2^8
    const int e = (int)(most >> 7) - 8 + ((most & 0x7fu) > 0x60u ? 1 : 0);
    return min(max(e, 127 - 117), 127 + 119);
}
// ... of a group of 32 elements, four lanes; 255 if there is an infinity or a NaN among them.
__device__ __forceinline__ int group_exponent(const u32x4 &x) {
    unsigned most = 0;   // largest magnitude, as the bits of a bf16
#pragma unroll
    for (int e = 0; e < 4; ++e) most = max(most, max(x[e] & 0x7fffu, (x[e] >> 16) & 0x7fffu));
    most = dpp_umax<0xB1>(most);    // quad_perm [1,0,3,2]
    most = dpp_umax<0x4E>(most);    // quad_perm [2,3,0,1]
    // most = 1.f * 2^(E - 127), and 7 = 1.75 * 2^2
    const int e = (int)(most >> 7) - 2 + ((most & 0x7fu) > 0x60u ? 1 : 0);
    return most >= 0x7f80u ? 255 : min(max(e, 127 - 125), 127 + 125);
}
// (the conversion divides by the power of two, rounds to the nearest, ties to the even code, and takes 6 for what is larger)
__device__ __forceinline__ unsigned pack_fp4(const u32x4 &x, int biased) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const float scale = power_of_two(biased);
    unsigned y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, __builtin_bit_cast(bf16x2, (unsigned)x[0]), scale, 0);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, __builtin_bit_cast(bf16x2, (unsigned)x[1]), scale, 1);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, __builtin_bit_cast(bf16x2, (unsigned)x[2]), scale, 2);
    y = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(y, __builtin_bit_cast(bf16x2, (unsigned)x[3]), scale, 3);
    return biased == 255 ? 0u : y;
}
__device__ __forceinline__ u32x2 pack_fp8(const u32x4 &x, int biased) {
    const float inverse = power_of_two(254 - biased);
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const unsigned b = e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16;
        const float z = __builtin_amdgcn_fmed3f(__builtin_bit_cast(float, b) * inverse, -448.f, 448.f);   // (exact, or below half of the least number)
        y[e] = (b & 0x7f800000u) == 0x7f800000u ? __builtin_nanf("") : z;
    }
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    return {(unsigned)lo, (unsigned)hi};
}

constexpr int PIECE_BYTES[] = {16, 8, 4};   // of 8 elements, by format
// where the exponents of a row (F4: of its first group) lie
template <int D, int F>
__device__ __forceinline__ int64_t exponent_at(const MoveArgs &a, const Place &p) {
    return ((((int64_t)p.page * a.n_kv_heads + p.head) << a.rows.shift) + p.slot) * (F == KSA_CACHE_FP4 ? D / 32 : 1);
}

// A row's piece of 8 elements of k and of v into the cache.
template <int D, int F>
__device__ __forceinline__ void put_piece(const MoveArgs &a, const Place &p, int piece, const u32x4 &k, const u32x4 &v) {
    constexpr int LANES = D / 8;
    const int64_t to = p.page * a.page_bytes + p.head * a.head_bytes + p.slot * a.row_bytes + piece * PIECE_BYTES[F];
    if constexpr (F == KSA_CACHE_FP8) {
        const int ke = row_exponent<LANES>(k), ve = row_exponent<LANES>(v);
        *reinterpret_cast<u32x2 *>(a.kc + to) = pack_fp8(k, ke);
        *reinterpret_cast<u32x2 *>(a.vc + to) = pack_fp8(v, ve);
        if (piece == 0) {
            const int64_t at = exponent_at<D, F>(a, p);
            a.k_exp[at] = (uint8_t)ke, a.v_exp[at] = (uint8_t)ve;
        }
    } else if constexpr (F == KSA_CACHE_FP4) {
        const int ke = group_exponent(k), ve = group_exponent(v);
        *reinterpret_cast<unsigned *>(a.kc + to) = pack_fp4(k, ke);
        *reinterpret_cast<unsigned *>(a.vc + to) = pack_fp4(v, ve);
        if (piece % 4 == 0) {
            const int64_t at = exponent_at<D, F>(a, p) + piece / 4;
            a.k_exp[at] = (uint8_t)ke, a.v_exp[at] = (uint8_t)ve;
        }
    } else {
        *reinterpret_cast<u32x4 *>(a.kc + to) = k;
        *reinterpret_cast<u32x4 *>(a.vc + to) = v;
    }
}

template <int D, int F>
__global__ __launch_bounds__(256) void ksa_paged_append_kernel(const MoveArgs a) {
    constexpr int LANES = D / 8;
    const int group = ksa_div(blockIdx.x, a.by_heads), head = blockIdx.x - group * a.n_kv_heads;
    const Place p = place_of<LANES>(a, group, head);
    if (p.page < 0) return;
    const int piece = threadIdx.x % LANES;
    const int64_t from = p.row * a.row_stride + p.head * a.head_stride + piece * 8;
    // (4 bits: what is read is four times what is written, and is not kept in the caches.  Kept and not kept (us), inputs in memory: 36864 rows in 50.7 and 42.8, in and out 83.4 and
    // 73.7, 8192 rows in 13.6 and 12.1, 2048 rows 5.0 and 5.3; inputs just made, with what makes them: 36864 rows in 87.5 and 89.0, in and out 139.9 and 126.9, 8192 rows in 22.8
    // and 24.4, in and out 31.8 and 32.0)
    auto load = [](const __bf16 *x) {
        const u32x4 *const at = reinterpret_cast<const u32x4 *>(x);
        if constexpr (F == KSA_CACHE_FP4) return __builtin_nontemporal_load(at);
        else return *at;
    };
    const u32x4 k = load(a.k + from), v = load(a.v + from);
    put_piece<D, F>(a, p, piece, k, v);
}

template <int D, int F>
__global__ __launch_bounds__(256) void ksa_paged_read_kernel(const MoveArgs a) {
    constexpr int LANES = D / 8;
    const int group = ksa_div(blockIdx.x, a.by_heads), head = blockIdx.x - group * a.n_kv_heads;
    const Place p = place_of<LANES>(a, group, head);
    if (!p.any) return;
    const int piece = threadIdx.x % LANES;
    u32x4 k = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u}, v = k;   // NaN
    if (p.page >= 0) {
        const int64_t from = p.page * a.page_bytes + p.head * a.head_bytes + p.slot * a.row_bytes + piece * PIECE_BYTES[F];
        if constexpr (F == KSA_CACHE_FP8) {
            const int64_t at = exponent_at<D, F>(a, p);
            const float ks = power_of_two(a.k_exp[at]), vs = power_of_two(a.v_exp[at]);
            const u32x2 x = *reinterpret_cast<const u32x2 *>(a.kc + from), y = *reinterpret_cast<const u32x2 *>(a.vc + from);
            const u32x2 k0 = unpack_fp8(x[0], ks), k1 = unpack_fp8(x[1], ks), v0 = unpack_fp8(y[0], vs), v1 = unpack_fp8(y[1], vs);
            k = u32x4{k0[0], k0[1], k1[0], k1[1]}, v = u32x4{v0[0], v0[1], v1[0], v1[1]};
        } else if constexpr (F == KSA_CACHE_FP4) {
            const int64_t at = exponent_at<D, F>(a, p) + piece / 4;
            const float ks = power_of_two(a.k_exp[at]), vs = power_of_two(a.v_exp[at]);
            k = unpack_fp4(*reinterpret_cast<const unsigned *>(a.kc + from), ks), v = unpack_fp4(*reinterpret_cast<const unsigned *>(a.vc + from), vs);
        } else {
            k = *reinterpret_cast<const u32x4 *>(a.kc + from), v = *reinterpret_cast<const u32x4 *>(a.vc + from);
        }
    }
    const int64_t to = p.row * a.row_stride + p.head * a.head_stride + piece * 8;
    *reinterpret_cast<u32x4 *>(a.k + to) = k;
    *reinterpret_cast<u32x4 *>(a.v + to) = v;
}

MoveArgs move_args(const KsaPagedMove &L) {
    MoveArgs a;
    a.rows = paged_rows(L.call);
    a.k = static_cast<__bf16 *>(L.k), a.v = static_cast<__bf16 *>(L.v);
    a.row_stride = L.strides[0], a.head_stride = L.strides[1];
    a.kc = static_cast<unsigned char *>(L.call.cache.k), a.vc = static_cast<unsigned char *>(L.call.cache.v);
    a.k_exp = L.call.cache.k_exp, a.v_exp = L.call.cache.v_exp;
    a.page_bytes = L.call.cache_strides[0], a.head_bytes = L.call.cache_strides[1], a.row_bytes = L.call.cache_strides[2];
    a.n_kv_heads = L.call.p.n_kv_heads;
    a.by_heads = ksa_divisor(a.n_kv_heads);
    return a;
}

// Blocks of a launch over all rows.
inline dim3 move_grid(const MoveArgs &a, int head_dim) {
    const int rows = 2048 / head_dim;
    return dim3((unsigned)((a.rows.total + rows - 1) / rows * a.n_kv_heads));
}

}  // namespace

#endif
