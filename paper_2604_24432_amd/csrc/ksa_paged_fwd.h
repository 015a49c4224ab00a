// Attention of new rows over the paged cache for gfx950: the kernels, of which every source makes those of its formats.
//
// o = sum_x w_x v_x / sum_x w_x, w_x = 2^(s_x - m) over the keys x that a row sees, s = log2(e) scale q k, m a reference of the row's.  Two kernels, each one
// pass over the keys, both products on the matrix unit with the keys as rows of the first and the (row, query head) pairs as its columns, so that a
// lane has its pair's weights where the second product wants them.  Few pairs of a KV head (ksa_paged_few_kernel): bound by the cache's bytes, so every wave
// streams blocks of 32 keys of its own, once for all pairs.  Many (ksa_paged_many_kernel): bound by the products, so a workgroup holds 128 or 256
// pairs, 32 per wave, and walks tiles of 64 keys that its waves share in LDS.  Either may cut the keys into spans, one workgroup each, whose
// records a third kernel joins by log-sum-exp.
//
// The keys that a group of rows sees together form one list, summaries first, then text (Eq. 3); where a position of the list lies is
// looked up in the tables a block ahead of its loads.  8-bit and 4-bit rows become bf16 on their way to the operands, exactly: the conversion takes the power
// of two along.
#ifndef KSA_PAGED_FWD_H_
#define KSA_PAGED_FWD_H_

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "ksa_paged.h"

namespace {

struct FwdArgs {
    PagedRows rows;
    const unsigned char *k, *v;
    const uint8_t *k_exp, *v_exp;
    int64_t page_bytes, head_bytes, row_bytes;   // strides of k and v
    const __bf16 *q;
    __bf16 *o;
    float *lse, *ws;
    int64_t q_row, q_head, o_row, o_head;
    int32_t max_rows;
    int32_t n_q_heads, n_kv_heads, group, n_splits;
    KsaDivisor by_group, by_heads, by_splits, by_q_heads;
    float q_scale, score_scale;   // scale * log2(e) in two factors, the first a power of two that goes into q
};

constexpr float LOWEST = -FLT_MAX;

// Largest exponent byte of the 8-bit format.  Where a key is not seen by every row a larger one of its V row counts as this one, so that the row is
// finite (448 * 2^119 is a bf16 number) and a weight of zero keeps it out of a sum.  Slots that were never written hold such bytes: what is read
// in a missing page's place, summaries that are listed and seen by no row, and rows that only others see.
constexpr int MOST_EXP = 127 + 119;
// ... of the 4-bit format (6 * 2^125 is a bf16 number), and the one of a group that is no numbers.
constexpr int MOST_EXP4 = 127 + 125, NO_NUMBERS = 255;

constexpr bool is_fp8(int format) { return format == KSA_CACHE_FP8; }
constexpr bool is_fp4(int format) { return format == KSA_CACHE_FP4; }
constexpr int bytes_of(int format, int elements) { return is_fp4(format) ? elements / 2 : is_fp8(format) ? elements : elements * 2; }
constexpr int PARTS[] = {1, 2};   // pieces of 8 bf16 that 16 bytes of a row become, by format

__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
    const unsigned lo = (unsigned)__shfl((int)(unsigned)x, lane), hi = (unsigned)__shfl((int)(unsigned)(x >> 32), lane);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

__device__ __forceinline__ int64_t spot_bytes(const FwdArgs &a, const Spot &s) { return max(s.page, 0) * a.page_bytes + s.slot * a.row_bytes; }
__device__ __forceinline__ int64_t spot_exp(const FwdArgs &a, const Spot &s, int hkv) {
    return (((int64_t)max(s.page, 0) * a.n_kv_heads + hkv) << a.rows.shift) + s.slot;
}

// Sixteen bytes of a cache row as bf16: 8 elements, or 16 of an 8-bit row.
template <int F>
__device__ __forceinline__ void as_bf16(const u32x4 &x, float scale, u32x4 (&y)[PARTS[F]]) {
    if constexpr (is_fp8(F)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const u32x2 z = unpack_fp8(x[e], scale);
            y[e / 2][2 * (e & 1)] = z[0], y[e / 2][2 * (e & 1) + 1] = z[1];
        }
    } else {
        y[0] = x;
    }
}

// V elements that are no numbers.  A weight of zero does not keep them out of a sum, so where not every row sees every key they are
// taken out of the product and added afterwards, to the rows that see them.
__device__ __forceinline__ bool take_out(unsigned &x) {
    const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
    x = (lo ? 0u : x & 0xffffu) | (hi ? 0u : x & 0xffff0000u);
    return lo || hi;
}
__device__ __forceinline__ bool take_out(u32x4 &x) {
    bool any = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        unsigned y = x[e];
        any |= take_out(y);
        x[e] = y;
    }
    return any;
}
// Bytes of an 8-bit word (halves of a word of bf16) that are no numbers become zero; whether there were any.
template <int F>
__device__ __forceinline__ bool take_out_raw(u32x4 &x) {
    if constexpr (!is_fp8(F)) return take_out(x);
    unsigned any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned hit = ((x[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;   // (0x7f and 0xff are the NaNs)
        any |= hit, x[e] &= ~((hit >> 7) * 0xffu);
    }
    return any != 0;
}

// A part of a 4-bit group that is no numbers becomes zeros; exponents beyond the largest count as that one.
template <int WORDS, class T>
__device__ __forceinline__ bool take_out_group(T &x, int &e) {
    const bool odd = e == NO_NUMBERS;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) x[i] = odd ? 0u : x[i];
    e = min(e, MOST_EXP4);
    return odd;
}

// four elements of a V row from column d on; those that are numbers are zero
template <int D, int F>
__device__ __forceinline__ void no_numbers(const FwdArgs &a, int hkv, const Spot &s, int d, float (&y)[4]) {
    if constexpr (is_fp4(F)) {
        const bool odd = a.v_exp[spot_exp(a, s, hkv) * (D / 32) + d / 32] == NO_NUMBERS;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = odd ? __builtin_nanf("") : 0.f;
        return;
    }
    const unsigned char *row = a.v + hkv * a.head_bytes + spot_bytes(a, s) + bytes_of(F, d);
    u32x2 x;
    if constexpr (is_fp8(F)) x = unpack_fp8(*reinterpret_cast<const unsigned *>(row), power_of_two(a.v_exp[spot_exp(a, s, hkv)]));
    else x = *reinterpret_cast<const u32x2 *>(row);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned z = e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16;
        y[e] = (z & 0x7f800000u) == 0x7f800000u ? __builtin_bit_cast(float, z) : 0.f;
    }
}

// an eighth of a row's elements of q times the power of two that goes into it
__device__ __forceinline__ bf16x8 scaled_q(const __bf16 *q, float by) {
    bf16x8 x = *reinterpret_cast<const bf16x8 *>(q);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (__bf16)((float)x[e] * by);
    return x;
}

__device__ __forceinline__ float log_sum(float m, float l) { return (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f; }

// Many rows: a row's reference is one of its scores, not always the largest: no weight is too small to count, and the sum of 16 of them is looked
// at instead of their scores.  Above this the largest becomes the reference and the 16 are worked out again.  In range 2^20 would do, but a weight of 1
// is exact in bf16 and the largest one's rounding is what the output keeps of all of them: off by 1.40 times an output's own rounding (4000 keys,
// half of the scores within 1), with 128 1.22, with 64 1.12.  Time: full attention of 2048 rows over 64K keys 1997 us with 2^20, 2029 with 128, 2067 with 64;
// window of 1023 30.2, 32.0, 33.2; a running maximum takes eight more vector instructions of a hundred in every half, 64 more where it moves.
// The sum is of the weights as they are in 32 bits, of which many average their roundings out; the sum of the rounded ones took 4 - 8 %.
constexpr float HIGH = 128.f;

// Bytes from one row of a tile to the next in LDS: the 16 rows of a phase of the plain reads of K, 16 bytes each, and the 4 rows of one of the
// transposing reads of V, 64 bytes each, lie in different banks, and every address is a base plus a constant.
template <int D>
struct TileRow {
    static constexpr int K = D * 2 + 16, V = D * 2 + 64;
};

// Sixteen weights of a lane that sum up to more than HIGH: the row's reference becomes the largest of its scores, what has been summed follows.
template <int DB>
__device__ __forceinline__ float raised(const f32x16 &sc, float sum, float m_run, float scale, float &l_run, f32x16 (&o)[DB]) {
    float most = sc[0];
#pragma unroll
    for (int g = 1; g < 16; ++g) most = fmaxf(most, sc[g]);
    most = fmaxf(most, other_half(most)) * scale;
    const float m = fmaxf(sum, other_half(sum)) > HIGH ? fmaxf(most, m_run) : m_run;   // (by the row alone)
    const float alpha = __builtin_amdgcn_exp2f(m_run - m);
    l_run *= alpha;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 16; ++g) o[db][g] *= alpha;
    return m;
}
// The scores of 32 keys where not all are seen by all: a lane's are those of keys 8 (g / 4) + 4 h + g % 4.  Bit i of `sees`: the row sees key i, of `none`:
// it has no page.  (Two vector instructions per score, from bits spread over words; comparing positions took twelve: a tile of 64 keys and 128 pairs
// alone on its unit 2.9 us, now 2.1; where all is seen 1.45.)
__device__ __forceinline__ void hide(f32x16 &sc, unsigned sees, unsigned none, int h) {
    const unsigned see = sees >> (4 * h), gone = none >> (4 * h);
    auto spread = [](unsigned x, int g) { return (unsigned)((int)(x << (31 - 8 * (g / 4) - g % 4)) >> 31); };   // all bits of a word
    auto choose = [](unsigned which, unsigned x, unsigned y) { return (which & x) | (~which & y); };
    if (none != 0) {
#pragma unroll
        for (int g = 0; g < 16; ++g) sc[g] = __builtin_bit_cast(float, choose(spread(gone, g), 0x7fc00000u, __builtin_bit_cast(unsigned, (float)sc[g])));
    }
#pragma unroll
    for (int g = 0; g < 16; ++g) sc[g] = __builtin_bit_cast(float, choose(spread(see, g), __builtin_bit_cast(unsigned, (float)sc[g]), 0xff800000u));
}
// The elements of a V row that are no numbers, to the output of a row that sees it.
template <int D, int F>
__device__ __forceinline__ void add_no_numbers(const FwdArgs &a, int hkv, const Spot &at, int h, bool see, f32x16 (&o)[D / 32]) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float z[4];
            no_numbers<D, F>(a, hkv, at, db * 32 + 8 * g + 4 * h, z);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][4 * g + e] += see ? z[e] : 0.f;
        }
}

// ---- few rows -----------------------------------------------------------------------------------------------------------

// At most 32 pairs.  Every wave has blocks of 32 keys of its own, in LDS of its own: no barriers before the end.  The rows of the next block are
// on their way while one is worked on: 64 KB per compute unit, two workgroups on each.  With one pair or 32 the work is the same, so the products cost
// nothing extra where there are few; references are running maxima.  64 sequences at 128K, 32/8 heads, 8-bit, 2.2 GB 334 us, bf16 634, 6.5 - 6.8 TB/s
// of the 6.8 that a plain read reaches: bound by HBM.  16 sequences of lengths 1 : 3, 8 rows each, 190 MB, 47 us in four spans: by the longest span and by
// 250 vector instructions per block, of which 8-bit rows' way to bf16 is 90 (bf16, twice the bytes, 72).  4 sequences, 25 MB 13.4 us in 16 spans of
// 120 keys: a chain of loads, entry, row, LDS.  One, 315 keys 6.3 us.  Dropped: keys of a tile shared by the waves, with two barriers for each (67 and
// 189 us for the 16 sequences' 8-bit and bf16), the sum of weights looked at as below (level, with outputs off by 1.35 times their own rounding
// instead of 1.1), weights in two bf16 parts (1.0, 8 % slower on 8-bit caches).
constexpr int FEW_WAVES = 4, BLOCK = 32;

template <int D, int F>
__global__ __launch_bounds__(FEW_WAVES * 64, 2) void ksa_paged_few_kernel(const FwdArgs a) {
    constexpr int KS = D / 16, DB = D / 32;
    constexpr int LPR = bytes_of(F, D) / 16, RPI = 64 / LPR, NI = BLOCK / RPI;   // lanes per row, rows per load, loads per tensor
    constexpr int KROW = TileRow<D>::K, VROW = TileRow<D>::V, OWN = BLOCK * (KROW + VROW), OUT_ROW = D + 4;
    static_assert(BLOCK * OUT_ROW * 4 <= OWN, "a wave's results lie where its blocks were");
    __shared__ __align__(16) unsigned char lds[FEW_WAVES * OWN];
    __shared__ float sh_m[FEW_WAVES][32], sh_l[FEW_WAVES][32];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 31, h = lane >> 5;
    const int split = blockIdx.x, hkv = blockIdx.y, b = blockIdx.z;
    const NewRows seq = new_rows(a.rows, b, a.max_rows);
    if (seq.n == 0) return;
    if (!seq.ok) {
        if (a.n_splits > 1) return;   // (the joining kernel sees to it)
        for (int x = tid / D; x < seq.n * a.group; x += FEW_WAVES * 64 / D) {
            const int row = x / a.group, hq = hkv * a.group + x % a.group;
            a.o[(seq.first + row) * a.o_row + hq * a.o_head + tid % D] = (__bf16)__builtin_nanf("");
            if (a.lse && tid % D == 0) a.lse[(int64_t)(seq.first + row) * a.n_q_heads + hq] = __builtin_nanf("");
        }
        return;
    }
    const Keys keys = keys_of(a.rows, seq.start, seq.start + seq.n - 1);
    const int per = ksa_div((keys.n + BLOCK - 1) / BLOCK + a.n_splits - 1, a.by_splits) * BLOCK;
    const int v0 = split * per, v1 = min(keys.n, v0 + per);

    // ---- blocks on their way: table entries two ahead, rows into registers one ahead, as bf16 into LDS ----------------------
    const unsigned char *const kb = a.k + hkv * a.head_bytes, *const vb = a.v + hkv * a.head_bytes;
    const int f_row = lane / LPR, f_piece = lane % LPR;
    u32x4 kr[NI], vr[NI];
    int ke = 0, ve = 0;        // exponents of row lane % 32
    unsigned lost = 0;         // keys without a page
    // Loads return in the order they are issued in: a block's table entries are asked for before the rows of the block in front of it.
    Entry entry;               // of row lane % 32 of the block to be requested next
    auto look = [&](int x) { return entry_of(a.rows, b, key_at(keys, min(x + r, keys.n - 1))); };
    auto request = [&](int x_next) {
        const Spot spot = spot_of(a.rows, entry);
        entry = look(x_next);
        const int64_t off = spot_bytes(a, spot);
        lost = (unsigned)__builtin_amdgcn_ballot_w64(spot.page < 0);
        if constexpr (is_fp8(F)) {
            const int64_t at = spot_exp(a, spot, hkv);
            ke = a.k_exp[at], ve = a.v_exp[at];
        }
        int64_t from[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) from[i] = lane_value(off, i * RPI + f_row) + f_piece * 16;
#pragma unroll
        for (int i = 0; i < NI; ++i) kr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kb + from[i]));
#pragma unroll
        for (int i = 0; i < NI; ++i) vr[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vb + from[i]));
    };
    constexpr int STEP = FEW_WAVES * BLOCK;
    const int first = v0 + wave * BLOCK;
    if (first < v1) {
        entry = look(first);
        request(first + STEP);
    }

    // the lane's pair = row * group + head (the last one repeats)
    const int pairs = seq.n * a.group, pair = min(r, pairs - 1), q_row = ksa_div(pair, a.by_group), q_head = hkv * a.group + pair - q_row * a.group;
    const Seen seen = seen_of(keys, visible(a.rows, kind_of(a.rows, seq.start + q_row)));
    bf16x8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = scaled_q(a.q + (seq.first + q_row) * a.q_row + q_head * a.q_head + s * 16 + h * 8, a.q_scale);

    f32x16 o[DB];
    float m_run = LOWEST, l_run = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 16; ++g) o[db][g] = 0.f;
    unsigned char *const own = lds + wave * OWN;
    const int grp = lane >> 4, li = lane & 15;
    const unsigned char *const k_at = own + r * KROW + h * 16;
    const unsigned char *const v_at = own + BLOCK * KROW + (4 * (grp >> 1) + (li >> 2)) * VROW + 32 * (grp & 1) + 8 * (li & 3);
    unsigned char *const put_k_at = own + f_row * KROW + f_piece * 16 * PARTS[F], *const put_v_at = own + BLOCK * KROW + f_row * VROW + f_piece * 16 * PARTS[F];
    auto put = [&](const u32x4 &x, int e, int i, unsigned char *to) {
        u32x4 y[PARTS[F]];
        as_bf16<F>(x, is_fp8(F) ? power_of_two(__shfl(e, i * RPI + f_row)) : 1.f, y);
#pragma unroll
        for (int z = 0; z < PARTS[F]; ++z) *reinterpret_cast<u32x4 *>(to + z * 16) = y[z];
    };
    auto sees_all = [&](int x) { return __builtin_amdgcn_ballot_w64(!seen.sees_all(x, x + BLOCK)) == 0; };
    bool ever = false;         // elements of V were taken out
    for (int x = first; x < v1; x += STEP) {
        const unsigned none = lost;
        const bool whole = none == 0 && sees_all(x);
        if (!whole) {
            if (is_fp8(F)) ve = min(ve, MOST_EXP);
            bool odd = false;
#pragma unroll
            for (int i = 0; i < NI; ++i) odd |= take_out_raw<F>(vr[i]);
            ever |= __builtin_amdgcn_ballot_w64(odd) != 0;
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) put(kr[i], ke, i, put_k_at + i * RPI * KROW);
#pragma unroll
        for (int i = 0; i < NI; ++i) put(vr[i], ve, i, put_v_at + i * RPI * VROW);
        if (x + STEP < v1) request(x + 2 * STEP);

        f32x16 sc;
#pragma unroll
        for (int g = 0; g < 16; ++g) sc[g] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(k_at + s * 32), q[s], sc, 0, 0, 0);
        if (!whole) hide(sc, seen.sees_32(x), none, h);
        bf16x8 p[2];
        float sum = 0.f;
        auto weights = [&]() {
            sum = 0.f;
#pragma unroll
            for (int g = 0; g < 16; ++g) {
                const float w = __builtin_amdgcn_exp2f(fmaf(sc[g], a.score_scale, -m_run));
                sum += w, p[g / 8][g % 8] = (__bf16)w;
            }
        };
        float most = sc[0];
#pragma unroll
        for (int g = 1; g < 16; ++g) most = fmaxf(most, sc[g]);
        most = fmaxf(most, other_half(most)) * a.score_scale;
        if (__builtin_amdgcn_ballot_w64(most > m_run) != 0) {
            const float m = fmaxf(most, m_run), alpha = __builtin_amdgcn_exp2f(m_run - m);
            m_run = m, l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int g = 0; g < 16; ++g) o[db][g] *= alpha;
        }
        weights();
        l_run += sum;
#pragma unroll
        for (int y = 0; y < 2 * DB; ++y) {   // 16 keys y / DB, columns 32 (y % DB) ..
            const unsigned char *at = v_at + y / DB * 16 * VROW + y % DB * 64;
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(at));
            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(at + 8 * VROW));
            const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
            o[y % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[y / DB], o[y % DB], 0, 0, 0);
        }
    }
    if (ever) {   // what was taken out of V, to the rows that see it
        for (int x = first; x < v1; x += STEP)
            for (int key = 0; key < min(BLOCK, keys.n - x); ++key) {
                const Spot at = spot_of(a.rows, entry_of(a.rows, b, key_at(keys, x + key)));
                if (sees_all(x) && at.page >= 0) continue;   // (where a page is missing the sum is none anyway)
                add_no_numbers<D, F>(a, hkv, at, h, seen.sees(x + key), o);
            }
    }

    // ---- the waves' results ------------------------------------------------------------------------------------------
    const float l = l_run + other_half(l_run);
    if (h == 0) sh_m[wave][r] = m_run, sh_l[wave][r] = l;
    float *const mine = reinterpret_cast<float *>(own);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4 *>(mine + r * OUT_ROW + db * 32 + 8 * g + 4 * h) = f32x4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
    __syncthreads();
    constexpr int LANES = D / 8;   // lanes per pair
#pragma unroll
    for (int x = tid / LANES; x < 32; x += FEW_WAVES * 64 / LANES) {
        if (x >= pairs) break;
        const int d0 = tid % LANES * 8;
        float M = sh_m[0][x];
#pragma unroll
        for (int y = 1; y < FEW_WAVES; ++y) M = fmaxf(M, sh_m[y][x]);
        float den = 0.f, out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = 0.f;
#pragma unroll
        for (int y = 0; y < FEW_WAVES; ++y) {
            const float w = __builtin_amdgcn_exp2f(sh_m[y][x] - M);
            const float *from = reinterpret_cast<const float *>(lds + y * OWN) + x * OUT_ROW + d0;
            den += sh_l[y][x] * w;
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] += from[e] * w;
        }
        const int row = seq.first + ksa_div(x, a.by_group), hq = hkv * a.group + x - ksa_div(x, a.by_group) * a.group;
        if (a.n_splits == 1) {
            bf16x8 z;
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = (__bf16)(out[e] / den);
            *reinterpret_cast<bf16x8 *>(a.o + row * a.o_row + hq * a.o_head + d0) = z;
            if (a.lse && d0 == 0) a.lse[(int64_t)row * a.n_q_heads + hq] = log_sum(M, den);
        } else {
            float *rec = a.ws + (((int64_t)row * a.n_q_heads + hq) * a.n_splits + split) * OUT_ROW;
#pragma unroll
            for (int e = 0; e < 8; e += 4) *reinterpret_cast<f32x4 *>(rec + d0 + e) = f32x4{out[e], out[e + 1], out[e + 2], out[e + 3]};
            if (d0 == 0) rec[D] = M, rec[D + 1] = den;
        }
    }
}

// ---- many rows ----------------------------------------------------------------------------------------------------------

constexpr int BN = 64;   // keys of a tile
#define KSA_FENCE() __builtin_amdgcn_sched_barrier(0)

// What a workgroup works on: pairs [first, first + PAIRS) of sequence b's new text rows (or summary rows), p = row * group + head.
struct Tile {
    int b, first;
    bool text;
    NewRows seq;
    int text0, n_text, n_sum;   // first new text row's index; how many new rows of either kind
};
template <int PAIRS>
__device__ __forceinline__ Tile tile_of(const FwdArgs &a, int slot) {
    const int lane = threadIdx.x & 63;
    Tile t;
    t.b = -1;
    auto tiles = [&](int rows) { return (int)(((int64_t)rows * a.group + PAIRS - 1) / PAIRS); };
    int before = 0;
    for (int base = 0; base < a.rows.batch; base += 64) {
        // every lane a sequence; its tiles, and those of the lanes up to it
        const int b = min(base + lane, a.rows.batch - 1);
        const NewRows s = new_rows(a.rows, b, a.max_rows);
        const int t0 = s.ok ? text_before(a.rows, s.start) : 0, n_t = s.ok ? text_before(a.rows, s.start + s.n) - t0 : s.n;
        const int of_text = tiles(n_t), mine = base + lane < a.rows.batch ? of_text + tiles(s.n - n_t) : 0;
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int y = __shfl_up(upto, d);
            upto += lane >= d ? y : 0;
        }
        upto += before;
        const uint64_t from = __builtin_amdgcn_ballot_w64(upto > slot);
        if (from) {
            const int at = __builtin_ctzll(from);
            auto get = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
            const int in = slot - get(upto - mine), split_at = get(of_text);
            t.b = base + at;
            t.text = in < split_at;
            t.first = (t.text ? in : in - split_at) * PAIRS;
            t.seq = {get(s.first), get(s.n), get(s.start), get(s.ok ? 1 : 0) != 0};
            t.text0 = get(t0), t.n_text = get(n_t), t.n_sum = t.seq.n - t.n_text;
            return t;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return t;
}

// A step works on one tile of keys in two halves of 32.  What a half does: the scores of its keys, the weights of the half before, and the
// product with V of the half before that, so that the matrix unit's and the vector unit's work do not wait for each other.
// GROUPS groups of NW waves, 32 pairs each.  Two groups have the same pairs, each half of the keys, and their results are put together in LDS.
// 2048 rows over 64K keys, 32/8 heads (8 waves) 1.98 - 2.15 ms, 1.0 - 1.1 PFLOP/s, of the 1.36 that a library product of 16384^3 reaches: seven vector
// and two LDS instructions per MFMA keep the board at its power cap (2.0 GHz) with the matrix unit busy half of the time; 4608 rows over 19000 keys, 8-bit, 1.02 -
// 1.11 ms.  8 waves take a tile from L2 half as often
// as 4 (2.29 ms).  With one wave per SIMD issue is the bound (a half has 100 vector, 16 matrix, 25 LDS instructions and 20 waits): 1.45 us per tile,
// two groups 0.85.  Start and end are 6 us: sequence, entries, rows and q one behind the other 3.2, the first tile 1.7, results 1.2.  Dropped: 64 pairs per
// wave with accumulators in AGPRs (one wave per SIMD, 2.96 ms), operands read further ahead (level), rows asked for half a step ahead (8 x 100 rows in
// one span 111 us, now 91).
template <int D, int F, int NW, int GROUPS>
__global__ __launch_bounds__(NW * GROUPS * 64, 2) void ksa_paged_many_kernel(const FwdArgs a) {
    constexpr int KS = D / 16, DB = D / 32, PAIRS = NW * 32;
    constexpr int RW = BN / NW;                                       // rows of a tile that a wave fetches
    // bytes of a row per lane and load; a wave's rows of 4 bits are one load (with 16 bytes half of the lanes would repeat the others': 4608 rows at 128K 1175 us, now 1033 - 1060)
    constexpr int EACH = is_fp4(F) ? D / (2 * NW) : 16;
    constexpr int LPR = bytes_of(F, D) / EACH, RPI = 64 / LPR < RW ? 64 / LPR : RW, NI = RW / RPI;   // lanes per row, rows per load, loads per wave and tensor
    constexpr int AS_BF16 = EACH * 2 * D / bytes_of(F, D);            // what they are as bf16
    typedef unsigned piece_t __attribute__((ext_vector_type(EACH / 4)));
    constexpr int KROW = TileRow<D>::K, VROW = TileRow<D>::V, K_BYTES = BN * KROW, V_BYTES = BN * VROW;
    constexpr int STAGE_ROW = D * 2 + 16;
    static_assert(RW % RPI == 0 && NI >= 1, "a wave's rows are whole loads");
    constexpr int OWN = 2 * (K_BYTES + V_BYTES);   // of a group: two buffers of K, two of V
    static_assert(NW * 32 * STAGE_ROW <= OWN && (GROUPS == 1 || NW * 64 * (16 * DB + 2) * 4 <= OWN), "the results pass through the tiles' memory");
    __shared__ __align__(16) unsigned char sh_tiles[GROUPS * OWN];
    // of the K tile: which of a wave's rows have no page; bit 31: of the V tile before: elements were taken out
    __shared__ __align__(16) unsigned sh_states[GROUPS][2][NW];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6) % NW, group = __builtin_amdgcn_readfirstlane(tid >> 6) / NW;
    const int r = lane & 31, h = lane >> 5;
    unsigned char *const lds = sh_tiles + group * OWN;
    unsigned (*const sh_state)[NW] = sh_states[group];
    // KV heads fastest: with a multiple of 8 of them the tiles of one share an L2
    const int rest = ksa_div(blockIdx.x, a.by_heads), hkv = blockIdx.x - rest * a.n_kv_heads;
    const int slot = ksa_div(rest, a.by_splits), split = rest - slot * a.n_splits;
    const Tile tile = tile_of<PAIRS>(a, slot);
    if (tile.b < 0) return;
    const NewRows seq = tile.seq;
    const int n_rows = tile.text ? tile.n_text : tile.n_sum;
    const int n_pairs = (int)min((int64_t)PAIRS, (int64_t)n_rows * a.group - tile.first);
    if (!seq.ok) {
        if (a.n_splits > 1) return;   // (the joining kernel sees to it)
        for (int x = tid; x < n_pairs * D; x += NW * GROUPS * 64) {
            const int pair = tile.first + x / D, row = pair / a.group, hq = hkv * a.group + pair % a.group;
            a.o[(seq.first + row) * a.o_row + hq * a.o_head + x % D] = (__bf16)__builtin_nanf("");
            if (a.lse && x % D == 0) a.lse[(int64_t)(seq.first + row) * a.n_q_heads + hq] = __builtin_nanf("");
        }
        return;
    }
    // rows of the tile by index of their kind
    const int base = tile.text ? tile.text0 : seq.start - tile.text0;
    auto row_at = [&](int pair) { return RowKind{tile.text, base + ksa_div(tile.first + min(pair, n_pairs - 1), a.by_group)}; };   // (the last one repeats)
    const Visible v_lo = visible(a.rows, row_at(0)), v_hi = visible(a.rows, row_at(n_pairs - 1));
    const Keys keys = keys_between(v_lo, v_hi);
    // what every row of the tile sees, and every row of the wave
    auto all_of = [&](const Visible &first, const Visible &last) { return seen_of(keys, Visible{last.lo_s, first.hi_s, last.lo_t, first.hi_t}); };
    const Seen tile_all = all_of(v_lo, v_hi), wave_all = all_of(visible(a.rows, row_at(wave * 32)), visible(a.rows, row_at(wave * 32 + 31)));
    const int n_tiles = (keys.n + BN - 1) / BN, per = ksa_div(n_tiles + a.n_splits - 1, a.by_splits);
    const int span = split * per, span_end = min(n_tiles, span + per), steps = max(span_end - span + GROUPS - 1, 0) / GROUPS;   // steps of any group
    const int first_tile = span + group * steps, end_tile = min(span_end, first_tile + steps);

    // packed row and query head of a pair
    auto place_of = [&](int pair, int &row, int &hq) {
        const RowKind k = row_at(pair);
        row = seq.first + row_of(a.rows, k) - seq.start;
        hq = hkv * a.group + tile.first + min(pair, n_pairs - 1) - (k.idx - base) * a.group;
    };
    int q_row, q_head;   // the lane's pair
    place_of(wave * 32 + r, q_row, q_head);
    const Seen seen = seen_of(keys, visible(a.rows, row_at(wave * 32 + r)));
    bf16x8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = scaled_q(a.q + q_row * a.q_row + q_head * a.q_head + s * 16 + h * 8, a.q_scale);

    // ---- tiles on their way: table entries three tiles ahead, rows into registers, then as bf16 into LDS; V a step behind K.  A row is asked for a
    // whole step before it goes to LDS: with one workgroup on a compute unit nothing else hides how long it takes. --------------------
    const unsigned char *const kb = a.k + hkv * a.head_bytes, *const vb = a.v + hkv * a.head_bytes;
    const int f_row = lane / LPR % RPI, f_piece = lane % LPR;   // (lanes beyond the rows repeat them)
    Entry entry;                               // of row RW * wave + lane % RW of a tile
    int64_t next_at = 0;                       // where that row of the next K tile lies
    int64_t exp_at = 0;                        // ... and its exponents
    static_assert(!is_fp4(F) || NI == 1, "4-bit rows: the exponents of the lane's one piece");
    int k_e = 0, v_e = 0, next_k_e = 0, next_v_e = 0;
    int64_t from[NI];                          // where the rows of the lane's loads lie: of the K tile asked for last, then of the V tile
    piece_t k_rows[NI], v_rows[NI];
    bool lost = false, next_lost = false, odd = false;   // row lane % RW of the K tile on its way has no page; elements of V were taken out
    const int last = min(keys.n, end_tile * BN) - 1;
    auto look = [&](int t) { entry = entry_of(a.rows, tile.b, key_at(keys, min(t * BN + RW * wave + lane % RW, last))); };
    auto settle = [&]() {
        const Spot spot = spot_of(a.rows, entry);
        next_lost = spot.page < 0;
        next_at = spot_bytes(a, spot);
        if constexpr (is_fp8(F)) exp_at = spot_exp(a, spot, hkv);
        if constexpr (is_fp4(F)) exp_at = lane_value(spot_exp(a, spot, hkv) * (D / 32), f_row) + f_piece * EACH / 16;
    };
    auto find = [&](int i) { from[i] = lane_value(next_at, i * RPI + f_row) + f_piece * EACH; };
    auto load_exps = [&]() {
        if constexpr (F != KSA_CACHE_BF16) next_k_e = a.k_exp[exp_at], next_v_e = a.v_exp[exp_at];
    };
    auto take_exps = [&]() {   // (a step after they were asked for)
        if constexpr (is_fp8(F)) k_e = next_k_e, v_e = min(next_v_e, MOST_EXP);
        if constexpr (is_fp4(F)) k_e = next_k_e, v_e = next_v_e;
    };
    auto load_k = [&](int i) { k_rows[i] = *reinterpret_cast<const piece_t *>(kb + from[i]); };
    auto load_v = [&](int i) { v_rows[i] = *reinterpret_cast<const piece_t *>(vb + from[i]); };
    auto put = [&](const piece_t &x, int e, int i, unsigned char *to) {
        if constexpr (is_fp4(F)) {
#pragma unroll
            for (int z = 0; z < EACH / 4; ++z) *reinterpret_cast<u32x4 *>(to + z * 16) = unpack_fp4(x[z], power_of_two(e));
        } else {
            u32x4 y[PARTS[F]];
            as_bf16<F>(x, is_fp8(F) ? power_of_two(__shfl(e, i * RPI + f_row)) : 1.f, y);
#pragma unroll
            for (int z = 0; z < PARTS[F]; ++z) *reinterpret_cast<u32x4 *>(to + z * 16) = y[z];
        }
    };
    const int put_k_at = (RW * wave + f_row) * KROW + f_piece * AS_BF16, put_v_at = 2 * K_BYTES + (RW * wave + f_row) * VROW + f_piece * AS_BF16;
    auto put_k = [&](int t, int i) { put(k_rows[i], k_e, i, lds + (t & 1) * K_BYTES + put_k_at + i * RPI * KROW); };
    auto put_v = [&](int t, int i) { put(v_rows[i], v_e, i, lds + (t & 1) * V_BYTES + put_v_at + i * RPI * VROW); };
    auto put_state = [&](int t) {   // with K tile t and V tile t - 1
        const unsigned none = (unsigned)__builtin_amdgcn_ballot_w64(lost) & ((1u << RW) - 1), taken = __builtin_amdgcn_ballot_w64(odd) != 0 ? 1u << 31 : 0u;
        if (lane == 0) sh_state[t & 1][wave] = none | taken;
    };

    f32x16 o[DB], sc[2];
    bf16x8 p[2][2];
    float m_run = LOWEST, l_run = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 16; ++g) o[db][g] = 0.f;
    unsigned any_state = 0, ever = 0;
    const int grp = lane >> 4, li = lane & 15;
    const int k_at = r * KROW + h * 16, v_at = 2 * K_BYTES + (4 * (grp >> 1) + (li >> 2)) * VROW + 32 * (grp & 1) + 8 * (li & 3);

    // Half y of step t.  SCORES: of keys 32 y .. of K tile t, into sc[y].  WEIGHTS: of sc[y ^ 1] (half 0: tile t - 1, half 1: tile t) into
    // p[y ^ 1].  OUT: V tile t - 1, keys 32 y .., times p[y].  A slot is one MFMA and what the vector unit does beside it, pinned by fences;
    // beside(x) is what slot x of the half does for the tiles on their way.
    constexpr int AHEAD = is_fp4(F) ? 2 : 3, AHEAD_V = 2;   // operands are read so many slots before the MFMAs that use them (4 bits: three 1 - 2 % slower)
    bf16x8 k[KS];
    auto read_k = [&](int t, int y, int x) { k[x] = *reinterpret_cast<const bf16x8 *>(lds + (t & 1) * K_BYTES + y * 32 * KROW + k_at + x * 32); };
    auto half = [&](int t, auto y_tag, auto scores_tag, auto weights_tag, auto out_tag, auto &&beside) {
        constexpr int y = decltype(y_tag)::value;
        constexpr bool SCORES = decltype(scores_tag)::value, WEIGHTS = decltype(weights_tag)::value, OUT = decltype(out_tag)::value;
        constexpr int EACH = 16 / (2 * KS);   // weights per slot
        static_assert(2 * DB == KS, "as many slots with V as with K");
        float ex[16], sum = 0.f;
        auto weight = [&](int slot) {   // the three steps of a weight lie in slots one after the other
            if constexpr (WEIGHTS) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const int g = (slot - 2) * EACH + i;
                    if (g >= 0 && g < 16) {
                        sum += ex[g];
                        if (g & 1) p[y ^ 1][g / 8][g % 8 - 1] = (__bf16)ex[g - 1], p[y ^ 1][g / 8][g % 8] = (__bf16)ex[g];
                        if (g % 8 == 7) asm volatile("" : "+v"(p[y ^ 1][g / 8]), "+v"(sum));   // (in this slot and not where it is used)
                    }
                }
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const int g = (slot - 1) * EACH + i;
                    if (g >= 0 && g < 16) {
                        ex[g] = __builtin_amdgcn_exp2f(ex[g]);
                        asm volatile("" : "+v"(ex[g]));
                    }
                }
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const int g = slot * EACH + i;
                    if (g < 16) {
                        ex[g] = fmaf(sc[y ^ 1][g], a.score_scale, -m_run);
                        asm volatile("" : "+v"(ex[g]));
                    }
                }
            }
        };
        bf16x8 v[2 * DB];
        const unsigned char *const from_v = lds + ((t - 1) & 1) * V_BYTES + y * 32 * VROW + v_at;
        auto read_v = [&](int x) {   // 16 keys x / DB, columns 32 (x % DB) ..
            if constexpr (OUT) {
                const unsigned char *at = from_v + x / DB * 16 * VROW + x % DB * 64;
                const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(at));
                const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(at + 8 * VROW));
                v[x] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        if constexpr (SCORES && y == 0) {   // (those of half 1 have been read in half 0)
#pragma unroll
            for (int x = 0; x < AHEAD; ++x) read_k(t, 0, x);
        }
        KSA_FENCE();
#pragma unroll
        for (int x = 0; x < KS; ++x) {
            if (x + AHEAD < KS) {
                if constexpr (SCORES) read_k(t, y, x + AHEAD);
            } else if (x + AHEAD < KS + AHEAD_V) {
                read_v(x + AHEAD - KS);
            }
            if constexpr (SCORES) {
                if (x == 0) {
#pragma unroll
                    for (int g = 0; g < 16; ++g) sc[y][g] = 0.f;
                }
                sc[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[x], q[x], sc[y], 0, 0, 0);
            }
            weight(x);
            beside(x);
            KSA_FENCE();
        }
#pragma unroll
        for (int x = 0; x < KS; ++x) {
            if (x + AHEAD_V < KS) read_v(x + AHEAD_V);
            else if (SCORES && y == 0) read_k(t, 1, x + AHEAD_V - KS);
            if constexpr (OUT) o[x % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[x], p[y][x / DB], o[x % DB], 0, 0, 0);
            weight(KS + x);
            beside(KS + x);
            KSA_FENCE();
        }
        if constexpr (SCORES && y == 0) {
#pragma unroll
            for (int x = AHEAD_V; x < AHEAD; ++x) read_k(t, 1, x);
        }
        weight(2 * KS), weight(2 * KS + 1);
        if constexpr (WEIGHTS) {
            if (__builtin_amdgcn_ballot_w64(sum > HIGH) != 0) {
                m_run = raised(sc[y ^ 1], sum, m_run, a.score_scale, l_run, o);
                sum = 0.f;
#pragma unroll
                for (int g = 0; g < 16; ++g) {
                    const float w = __builtin_amdgcn_exp2f(fmaf(sc[y ^ 1][g], a.score_scale, -m_run));
                    sum += w, p[y ^ 1][g / 8][g % 8] = (__bf16)w;
                }
            }
            l_run += sum;
        }
        if constexpr (SCORES) {
            const int x0 = t * BN + 32 * y;
            if (!wave_all.sees_all(x0, x0 + 32) || any_state != 0) {
                unsigned none = 0;   // keys without a page
#pragma unroll
                for (int x = 0; x < NW / 2; ++x) none |= (sh_state[t & 1][y * (NW / 2) + x] & ((1u << RW) - 1)) << (x * RW);
                hide(sc[y], seen.sees_32(x0), none, h);
            }
        }
    };
    using Yes = std::true_type;
    using No = std::false_type;
    const std::integral_constant<int, 0> y0;
    const std::integral_constant<int, 1> y1;
    // Slots of a half: KS, and as many again.  Half 0 brings V of this tile to LDS and asks for the next, half 1 K of the next tile and asks
    // for the one after that; where its rows are, is worked out on the way.
    auto bring_v = [&](int t) {
        return [&, t](int x) {
            if (x == 2 * KS - NI) {
                odd = false;
                if (!tile_all.sees_all(t * BN, t * BN + BN)) {
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        if constexpr (is_fp4(F)) odd |= take_out_group<EACH / 4>(v_rows[i], v_e);
                        else odd |= take_out_raw<F>(v_rows[i]);
                    }
                }
            }
            if (x >= 2 * KS - NI) put_v(t, x - (2 * KS - NI)), load_v(x - (2 * KS - NI));
        };
    };
    auto bring_k = [&](int t) {
        return [&, t](int x) {
            if (x == 0) take_exps();
            if (x == 1) settle();
            if (x == 2) look(t + 2);
            if (x == 3) load_exps();
            if (x >= 4 && x < 4 + NI) find(x - 4);
            if (x == 2 * KS - NI) put_state(t), lost = next_lost;
            if (x >= 2 * KS - NI) put_k(t, x - (2 * KS - NI)), load_k(x - (2 * KS - NI));
        };
    };
    static_assert(4 + 2 * NI <= 2 * KS, "in one half");
    auto nothing = [](int) {};
    auto begin = [&](int t) {
        __syncthreads();
        unsigned state = 0;
#pragma unroll
        for (int x = 0; x < NW; x += 4) {
            const u32x4 four = *reinterpret_cast<const u32x4 *>(sh_state[t & 1] + x);
            state |= four[0] | four[1] | four[2] | four[3];
        }
        any_state = __builtin_amdgcn_readfirstlane(state);
        ever |= any_state;
    };

    if (first_tile < end_tile) {
        look(first_tile);
        settle();
        lost = next_lost;
        look(first_tile + 1);
        load_exps();
#pragma unroll
        for (int i = 0; i < NI; ++i) find(i), load_k(i);
#pragma unroll
        for (int i = 0; i < NI; ++i) load_v(i);
        take_exps();
#pragma unroll
        for (int i = 0; i < NI; ++i) put_k(first_tile, i);
        put_state(first_tile);
        settle();
        lost = next_lost;
        look(first_tile + 2);
        load_exps();
#pragma unroll
        for (int i = 0; i < NI; ++i) find(i), load_k(i);
        begin(first_tile);
        half(first_tile, y0, Yes{}, No{}, No{}, bring_v(first_tile));
        half(first_tile, y1, Yes{}, Yes{}, No{}, bring_k(first_tile + 1));
        for (int t = first_tile + 1; t < end_tile; ++t) {
            begin(t);
            half(t, y0, Yes{}, Yes{}, Yes{}, bring_v(t));
            half(t, y1, Yes{}, Yes{}, Yes{}, bring_k(t + 1));
        }
        begin(end_tile);
        half(end_tile, y0, No{}, Yes{}, Yes{}, nothing);
        half(end_tile, y1, No{}, No{}, Yes{}, nothing);
    }
    if constexpr (GROUPS > 1) {   // as many barriers in every group
        for (int t = max(end_tile - first_tile, 0); t < steps; ++t) __syncthreads();
        if (end_tile <= first_tile && steps > 0) __syncthreads();
    }

    // ---- results ---------------------------------------------------------------------------------------------------------
    if (ever >> 31) {   // what was taken out of V, to the rows that see it
#pragma unroll 1
        for (int x = first_tile * BN; x < min(end_tile * BN, keys.n); ++x) {
            if (tile_all.sees_all(x / BN * BN, x / BN * BN + BN)) continue;
            add_no_numbers<D, F>(a, hkv, spot_of(a.rows, entry_of(a.rows, tile.b, key_at(keys, x))), h, seen.sees(x), o);
        }
    }
    float l = l_run + other_half(l_run);
    if constexpr (GROUPS > 1) {
        float *const other = reinterpret_cast<float *>(sh_tiles + OWN) + wave * 64 * (16 * DB + 2) + lane;   // of the lane with the same pair
        __syncthreads();
        if (group == 1) {
#pragma unroll
            for (int x = 0; x < 16 * DB; ++x) other[x * 64] = o[x / 16][x % 16];
            other[16 * DB * 64] = m_run, other[(16 * DB + 1) * 64] = l;
        }
        __syncthreads();
        if (group == 1) return;
        const float m = other[16 * DB * 64], M = fmaxf(m_run, m), w = __builtin_amdgcn_exp2f(m_run - M), v = __builtin_amdgcn_exp2f(m - M);
#pragma unroll
        for (int x = 0; x < 16 * DB; ++x) o[x / 16][x % 16] = o[x / 16][x % 16] * w + other[x * 64] * v;
        l = l * w + other[(16 * DB + 1) * 64] * v, m_run = M;
    }
    const bool mine = wave * 32 + r < n_pairs;
    if (a.n_splits > 1) {
        if (!mine) return;
        float *rec = a.ws + (((int64_t)q_row * a.n_q_heads + q_head) * a.n_splits + split) * (D + 4);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4 *>(rec + db * 32 + 8 * g + 4 * h) = f32x4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
        if (h == 0) rec[D] = m_run, rec[D + 1] = l;
        return;
    }
    if (a.lse && h == 0 && mine) a.lse[(int64_t)q_row * a.n_q_heads + q_head] = log_sum(m_run, l);
    // whole rows are stored: through memory of the wave's own, where the tiles were
    if constexpr (GROUPS == 1) __syncthreads();
    unsigned char *const stage = lds + wave * 32 * STAGE_ROW;
    const float inv = 1.f / l;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            bf16x4 z;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = (__bf16)(o[db][4 * g + e] * inv);
            *reinterpret_cast<bf16x4 *>(stage + r * STAGE_ROW + (db * 32 + 8 * g + 4 * h) * 2) = z;
        }
    constexpr int OUT_LANES = D / 8, OUT_ROWS = 64 / OUT_LANES;
#pragma unroll
    for (int i = 0; i < 32 / OUT_ROWS; ++i) {
        const int at = i * OUT_ROWS + lane / OUT_LANES;
        const u32x4 z = *reinterpret_cast<const u32x4 *>(stage + at * STAGE_ROW + lane % OUT_LANES * 16);
        int to_row, to_head;
        place_of(wave * 32 + at, to_row, to_head);
        if (wave * 32 + at < n_pairs) *reinterpret_cast<u32x4 *>(a.o + to_row * a.o_row + to_head * a.o_head + lane % OUT_LANES * 8) = z;
    }
}

FwdArgs fwd_args(const KsaPagedFwd &L) {
    FwdArgs a;
    const ksa_params &p = L.call.p;
    a.rows = paged_rows(L.call);
    a.k = static_cast<const unsigned char *>(L.call.cache.k), a.v = static_cast<const unsigned char *>(L.call.cache.v);
    a.k_exp = L.call.cache.k_exp, a.v_exp = L.call.cache.v_exp;
    a.page_bytes = L.call.cache_strides[0], a.head_bytes = L.call.cache_strides[1], a.row_bytes = L.call.cache_strides[2];
    a.q = static_cast<const __bf16 *>(L.q), a.o = static_cast<__bf16 *>(L.o), a.lse = L.lse, a.ws = L.workspace;
    a.q_row = L.q_strides[0], a.q_head = L.q_strides[1], a.o_row = L.o_strides[0], a.o_head = L.o_strides[1];
    a.max_rows = L.max_rows;
    a.n_q_heads = p.n_q_heads, a.n_kv_heads = p.n_kv_heads, a.group = p.n_q_heads / p.n_kv_heads;
    a.n_splits = L.plan.n_splits;
    a.by_group = ksa_divisor(a.group), a.by_heads = ksa_divisor(a.n_kv_heads), a.by_splits = ksa_divisor(a.n_splits), a.by_q_heads = ksa_divisor(a.n_q_heads);
    // With the first factor in q the products are no larger than the scaled scores and at least half as large, so that they do not
    // overflow where those would not.
    const float scale = p.softmax_scale * 1.4426950408889634f;
    int exponent = 0;
    (void)std::frexp(scale, &exponent);
    a.q_scale = std::ldexp(1.f, std::max(std::min(exponent - 1, 0), -8)), a.score_scale = scale / a.q_scale;
    return a;
}

// (the spans' records, where there are several, are joined by ksa_launch_paged_join)
template <int D, int F>
void launch_many(const FwdArgs &a, const KsaPagedPlan &plan, hipStream_t st) {
    const dim3 many((unsigned)(plan.slots * plan.n_splits * a.n_kv_heads));
    if (plan.groups == 2) hipLaunchKernelGGL((ksa_paged_many_kernel<D, F, 4, 2>), many, dim3(512), 0, st, a);
    else if (plan.pairs == 128) hipLaunchKernelGGL((ksa_paged_many_kernel<D, F, 4, 1>), many, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((ksa_paged_many_kernel<D, F, 8, 1>), many, dim3(512), 0, st, a);
}
template <int D, int F>
void launch_few(const FwdArgs &a, const KsaPagedPlan &plan, hipStream_t st) {
    hipLaunchKernelGGL((ksa_paged_few_kernel<D, F>), dim3(plan.n_splits, a.n_kv_heads, a.rows.batch), dim3(FEW_WAVES * 64), 0, st, a);
}

}  // namespace

#endif
