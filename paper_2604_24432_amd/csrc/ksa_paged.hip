// Attention of new rows over the paged cache for gfx950.
//
// Two kernels.  Few (row, query head) pairs of a KV head (ksa_paged_few_kernel): every wave streams blocks of 32 keys of its own, K from HBM
// into the registers of the score product's operand, V through LDS, once for all pairs.  Many (ksa_paged_many_kernel): a workgroup holds 128
// pairs, 32 per wave, and walks tiles of 64 keys that its waves share in LDS.  Either may cut the keys into spans, one workgroup each,
// whose records a third kernel joins by log-sum-exp.
//
// The keys that a group of rows sees together form one list, summaries first, then text (Eq. 3); where a position of the list lies is
// looked up in the tables a block ahead of its loads.  8-bit rows become bf16 on their way to the operands, exactly: the conversion takes the power
// of two along.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>

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
    KsaDivisor by_group, by_heads, by_splits;
    float q_scale, score_scale;   // scale * log2(e) in two factors, the first a power of two that goes into q
};

constexpr float LOWEST = -FLT_MAX;

// values of lane l ^ 16 and l ^ 32
__device__ __forceinline__ float swap16(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 16) ? r[0] : r[1]);
}
__device__ __forceinline__ float swap32(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}
__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
    const unsigned lo = (unsigned)__shfl((int)(unsigned)x, lane), hi = (unsigned)__shfl((int)(unsigned)(x >> 32), lane);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

__device__ __forceinline__ int64_t spot_bytes(const FwdArgs &a, const Spot &s) { return max(s.page, 0) * a.page_bytes + s.slot * a.row_bytes; }
__device__ __forceinline__ int64_t spot_exp(const FwdArgs &a, const Spot &s, int hkv) {
    return (((int64_t)max(s.page, 0) * a.n_kv_heads + hkv) << a.rows.shift) + s.slot;
}

// Sixteen bytes of a cache row as bf16: 8 elements, or 16 of an 8-bit row.
template <bool F8>
__device__ __forceinline__ void as_bf16(const u32x4 &x, float scale, u32x4 (&y)[F8 ? 2 : 1]) {
    if constexpr (F8) {
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
// four elements of a V row from column d on; those that are numbers are zero
template <bool F8>
__device__ __forceinline__ void no_numbers(const FwdArgs &a, int hkv, const Spot &s, int d, float (&y)[4]) {
    const unsigned char *row = a.v + hkv * a.head_bytes + spot_bytes(a, s) + d * (F8 ? 1 : 2);
    u32x2 x;
    if constexpr (F8) x = unpack_fp8(*reinterpret_cast<const unsigned *>(row), power_of_two(a.v_exp[spot_exp(a, s, hkv)]));
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

// ---- few rows -----------------------------------------------------------------------------------------------------------

constexpr int FEW_WAVES = 4, BLOCK = 32;   // keys of a wave's step

// The 16-byte pieces of a V row in LDS are dealt by this function of the row: the 8 rows that two groups of 16 lanes read 32 bytes of each
// (transposing reads) lie in different banks.
template <int D>
__device__ __forceinline__ int few_swz(int row) { return (D == 128 ? (row & 3) << 2 : (row & 2) << 1) ^ ((row & 4) >> 1); }

template <int D, bool F8, int NC>
__global__ __launch_bounds__(FEW_WAVES * 64) void ksa_paged_few_kernel(const FwdArgs a) {
    constexpr int CB = NC / 16, KS = D / 32, DB = D / 16, ES = F8 ? 1 : 2;
    constexpr int KL = D * ES / 64;          // loads per 16 keys of K: 64 bytes of each
    constexpr int LPR = D * ES / 16;         // lanes per V row
    constexpr int RPW = 64 / LPR, VL = BLOCK / RPW;
    constexpr int OUT_ROW = D + 4;
    __shared__ __align__(16) unsigned char lds[FEW_WAVES * 16 * OUT_ROW * 4];
    __shared__ float sh_m[FEW_WAVES][NC], sh_l[FEW_WAVES][NC];
    static_assert(FEW_WAVES * 16 * OUT_ROW * 4 >= FEW_WAVES * BLOCK * D * 2, "the results lie where the V blocks were");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int split = blockIdx.x, hkv = blockIdx.y, b = blockIdx.z;
    const NewRows seq = new_rows(a.rows, b, a.max_rows);
    if (seq.n == 0) return;
    if (!seq.ok) {
        if (a.n_splits > 1) return;   // (the joining kernel sees to it)
        for (int x = tid; x < seq.n * a.group * D; x += FEW_WAVES * 64) {
            const int row = x / (a.group * D), h = hkv * a.group + x / D % a.group;
            a.o[(seq.first + row) * a.o_row + h * a.o_head + x % D] = (__bf16)__builtin_nanf("");
            if (a.lse && x % D == 0) a.lse[(int64_t)(seq.first + row) * a.n_q_heads + h] = __builtin_nanf("");
        }
        return;
    }
    const Keys keys = keys_of(a.rows, seq.start, seq.start + seq.n - 1);
    const int blocks = (keys.n + BLOCK - 1) / BLOCK, per = ksa_div(blocks + a.n_splits - 1, a.by_splits) * BLOCK;
    const int v0 = split * per, v1 = min(keys.n, v0 + per);

    // pair p = row * group + head, of which column p % 16 of block p / 16 is this lane's (the last one repeats)
    const int pairs = seq.n * a.group;
    bf16x8 q[CB][KS];
    Seen seen[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int p = min(cb * 16 + col, pairs - 1), row = ksa_div(p, a.by_group), h = hkv * a.group + p - row * a.group;
        const __bf16 *from = a.q + (seq.first + row) * a.q_row + h * a.q_head;
#pragma unroll
        for (int s = 0; s < KS; ++s)   // (the columns of a step's operand are those that the lane has of a K row)
            q[cb][s] = scaled_q(from + (F8 ? (s / 2) * 64 + grp * 16 + (s & 1) * 8 : s * 32 + grp * 8), a.q_scale);
        seen[cb] = seen_of(keys, visible(a.rows, kind_of(a.rows, seq.start + row)));
    }
    f32x4 o[CB][DB];
    float m_run[CB], l_run[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        m_run[cb] = LOWEST, l_run[cb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[cb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    unsigned char *const vt = lds + wave * BLOCK * D * 2;
    const unsigned char *kb = a.k + hkv * a.head_bytes, *vb = a.v + hkv * a.head_bytes;
    const int t_row = 4 * grp + (col >> 2);
    const int t_at = t_row * (D * 2) + ((((col & 3) >> 1) ^ few_swz<D>(t_row)) << 4) + ((col & 1) << 3);

    const int step = FEW_WAVES * BLOCK;
    int x = v0 + wave * BLOCK;
    Spot next = spot_of(a.rows, b, key_at(keys, min(x + (lane & 31), keys.n - 1)));
    for (; x < v1; x += step) {
        const Spot spot = next;
        next = spot_of(a.rows, b, key_at(keys, min(x + step + (lane & 31), keys.n - 1)));
        const int64_t off = spot_bytes(a, spot);
        const unsigned lost = (unsigned)__builtin_amdgcn_ballot_w64(spot.page < 0);   // keys without a page
        int ke = 0, ve = 0;
        if constexpr (F8) {
            const int64_t at = spot_exp(a, spot, hkv);
            ke = a.k_exp[at], ve = a.v_exp[at];
        }
        u32x4 kk[2][KL], vv[VL];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const unsigned char *row = kb + lane_value(off, y * 16 + col) + grp * 16;
#pragma unroll
            for (int s = 0; s < KL; ++s) kk[y][s] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(row + s * 64));
        }
#pragma unroll
        for (int u = 0; u < VL; ++u)
            vv[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vb + lane_value(off, u * RPW + lane / LPR) + lane % LPR * 16));

        bool whole = lost == 0;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) whole &= seen[cb].sees_all(x, x + BLOCK);
        whole = __builtin_amdgcn_ballot_w64(!whole) == 0;

        f32x4 acc[2][CB];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const float scale = F8 ? power_of_two(__shfl(ke, y * 16 + col)) : 1.f;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) acc[y][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KL; ++s) {
                u32x4 ka[F8 ? 2 : 1];
                as_bf16<F8>(kk[y][s], scale, ka);
#pragma unroll
                for (int z = 0; z < (F8 ? 2 : 1); ++z)
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb)
                        acc[y][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ka[z]), q[cb][F8 ? 2 * s + z : s], acc[y][cb], 0, 0, 0);
            }
        }
        bool odd = false;   // elements were taken out
#pragma unroll
        for (int u = 0; u < VL; ++u) {
            u32x4 y[F8 ? 2 : 1];
            const int row = u * RPW + lane / LPR;
            as_bf16<F8>(vv[u], F8 ? power_of_two(__shfl(ve, row)) : 1.f, y);
#pragma unroll
            for (int z = 0; z < (F8 ? 2 : 1); ++z) {
                if (!whole) odd |= take_out(y[z]);
                const int piece = lane % LPR * (F8 ? 2 : 1) + z;
                *reinterpret_cast<u32x4 *>(vt + row * (D * 2) + ((piece ^ few_swz<D>(row)) << 4)) = y[z];
            }
        }
        odd = __builtin_amdgcn_ballot_w64(odd) != 0;

        bf16x8 p[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            float s[8], mx = LOWEST;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[e] = acc[e / 4][cb][e % 4] * a.score_scale;
                if (!whole) {
                    const int key = (e / 4) * 16 + grp * 4 + e % 4;
                    s[e] = !seen[cb].sees(x + key) ? -INFINITY : (lost >> key) & 1 ? __builtin_nanf("") : s[e];
                }
                mx = fmaxf(mx, s[e]);
            }
            if (__builtin_amdgcn_ballot_w64(mx > m_run[cb]) != 0) {
                mx = fmaxf(mx, swap16(mx));
                mx = fmaxf(fmaxf(mx, swap32(mx)), m_run[cb]);
                const float alpha = __builtin_amdgcn_exp2f(m_run[cb] - mx);
                m_run[cb] = mx, l_run[cb] *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db) o[cb][db] *= alpha;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float w = __builtin_amdgcn_exp2f(s[e] - m_run[cb]);
                l_run[cb] += w;
                p[cb][e] = (__bf16)w;
            }
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const unsigned char *at = vt + (t_at ^ (db << 5));
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(at));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(at + 16 * D * 2));
            const bf16x8 va = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) o[cb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, p[cb], o[cb][db], 0, 0, 0);
        }
        if (odd) {
            for (int key = 0; key < BLOCK; ++key) {
                const Spot at = {__builtin_amdgcn_readlane(spot.page, key), __builtin_amdgcn_readlane(spot.slot, key)};
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    float y[4];
                    no_numbers<F8>(a, hkv, at, db * 16 + grp * 4, y);
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[cb][db][e] += seen[cb].sees(x + key) ? y[e] : 0.f;
                }
            }
        }
    }

    // ---- the waves' results ------------------------------------------------------------------------------------------
    float *const sh_o = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        float l = l_run[cb];
        l += swap16(l), l += swap32(l);
        if (grp == 0) sh_m[wave][cb * 16 + col] = m_run[cb], sh_l[wave][cb * 16 + col] = l;
        __syncthreads();   // (the V blocks, or the results of the columns before, have been read)
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(sh_o + (wave * 16 + col) * OUT_ROW + db * 16 + grp * 4) = o[cb][db];
        __syncthreads();
        constexpr int EACH = D / 16;
        const int c = tid / 16, d0 = tid % 16 * EACH, pair = cb * 16 + c;
        if (pair < pairs) {
            float M = sh_m[0][pair];
#pragma unroll
            for (int y = 1; y < FEW_WAVES; ++y) M = fmaxf(M, sh_m[y][pair]);
            float den = 0.f, out[EACH];
#pragma unroll
            for (int e = 0; e < EACH; ++e) out[e] = 0.f;
#pragma unroll
            for (int y = 0; y < FEW_WAVES; ++y) {
                const float w = __builtin_amdgcn_exp2f(sh_m[y][pair] - M);
                den += sh_l[y][pair] * w;
#pragma unroll
                for (int e = 0; e < EACH; ++e) out[e] += sh_o[(y * 16 + c) * OUT_ROW + d0 + e] * w;
            }
            const int row = seq.first + ksa_div(pair, a.by_group), h = hkv * a.group + pair - ksa_div(pair, a.by_group) * a.group;
            if (a.n_splits == 1) {
                typedef __bf16 bf16_each __attribute__((ext_vector_type(EACH)));
                bf16_each r;
#pragma unroll
                for (int e = 0; e < EACH; ++e) r[e] = (__bf16)(out[e] / den);
                *reinterpret_cast<bf16_each *>(a.o + row * a.o_row + h * a.o_head + d0) = r;
                if (a.lse && d0 == 0) a.lse[(int64_t)row * a.n_q_heads + h] = log_sum(M, den);
            } else {
                float *rec = a.ws + (((int64_t)row * a.n_q_heads + h) * a.n_splits + split) * OUT_ROW;
#pragma unroll
                for (int e = 0; e < EACH; e += 4) *reinterpret_cast<f32x4 *>(rec + d0 + e) = f32x4{out[e], out[e + 1], out[e + 2], out[e + 3]};
                if (d0 == 0) rec[D] = M, rec[D + 1] = den;
            }
        }
    }
}

// ---- many rows ----------------------------------------------------------------------------------------------------------

constexpr int NW = 4, BN = 64, RW = BN / NW;   // waves; keys of a tile; rows of it that a wave fetches
static_assert(KSA_PAGED_PAIRS == NW * 32, "32 pairs per wave");

template <int D>
__device__ __forceinline__ int k_swz(int row) { return D == 64 ? (row >> 1) & 7 : row & (D / 8 - 1); }
template <int D>
__device__ __forceinline__ int v_swz(int row) { return D == 64 ? (row & 2) << 1 : ((row & 3) << 2) & (D / 8 - 1); }

// What a workgroup works on: pairs [first, first + 128) of sequence b's new text rows (or summary rows), p = row * group + head.
struct Tile {
    int b, first;
    bool text;
    NewRows seq;
    int text0, n_text, n_sum;   // first new text row's index; how many new rows of either kind
};
__device__ __forceinline__ Tile tile_of(const FwdArgs &a, int slot) {
    const int lane = threadIdx.x & 63;
    Tile t;
    t.b = -1;
    auto tiles = [&](int rows) { return (int)(((int64_t)rows * a.group + KSA_PAGED_PAIRS - 1) / KSA_PAGED_PAIRS); };
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
            t.first = (t.text ? in : in - split_at) * KSA_PAGED_PAIRS;
            t.seq = {get(s.first), get(s.n), get(s.start), get(s.ok ? 1 : 0) != 0};
            t.text0 = get(t0), t.n_text = get(n_t), t.n_sum = t.seq.n - t.n_text;
            return t;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return t;
}

template <int D, bool F8>
__global__ __launch_bounds__(NW * 64, 2) void ksa_paged_many_kernel(const FwdArgs a) {
    constexpr int KS = D / 16, DB = D / 32, ES = F8 ? 1 : 2;
    constexpr int LPR = D * ES / 16, RPI = 64 / LPR, NI = RW / RPI;   // lanes per row, rows per load, loads per wave and tensor
    constexpr int BYTES = BN * D * 2;
    static_assert(RW % RPI == 0 && NI >= 1, "a wave's rows are whole loads");
    __shared__ __align__(16) unsigned char lds[4 * BYTES];   // two buffers of K, then V
    __shared__ uint64_t sh_lost[2];                          // tile's keys without a page
    __shared__ int sh_odd[2][NW];                            // elements of V were taken out

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 31, h = lane >> 5;
    // KV heads fastest: with a multiple of 8 of them the tiles of one share an L2
    const int rest = ksa_div(blockIdx.x, a.by_heads), hkv = blockIdx.x - rest * a.n_kv_heads;
    const int slot = ksa_div(rest, a.by_splits), split = rest - slot * a.n_splits;
    const Tile tile = tile_of(a, slot);
    if (tile.b < 0) return;
    const NewRows seq = tile.seq;
    const int n_rows = tile.text ? tile.n_text : tile.n_sum;
    const int64_t all_pairs = (int64_t)n_rows * a.group;
    const int n_pairs = (int)min((int64_t)KSA_PAGED_PAIRS, all_pairs - tile.first);
    if (!seq.ok) {
        if (a.n_splits > 1) return;
        for (int x = tid; x < n_pairs * D; x += NW * 64) {
            const int pair = tile.first + x / D, row = pair / a.group, hq = hkv * a.group + pair % a.group;
            a.o[(seq.first + row) * a.o_row + hq * a.o_head + x % D] = (__bf16)__builtin_nanf("");
            if (a.lse && x % D == 0) a.lse[(int64_t)(seq.first + row) * a.n_q_heads + hq] = __builtin_nanf("");
        }
        return;
    }
    // rows of the tile by index of their kind
    const int sum0 = seq.start - tile.text0, base = tile.text ? tile.text0 : sum0;
    const int lo = base + ksa_div(tile.first, a.by_group), hi = base + ksa_div(tile.first + n_pairs - 1, a.by_group);
    const RowKind r_lo = {tile.text, lo}, r_hi = {tile.text, hi};
    const Visible v_lo = visible(a.rows, r_lo), v_hi = visible(a.rows, r_hi);
    const Keys keys = keys_between(v_lo, v_hi);
    // what every row of the tile sees
    const Seen every = seen_of(keys, Visible{v_hi.lo_s, v_lo.hi_s, v_hi.lo_t, v_lo.hi_t});
    const int n_tiles = (keys.n + BN - 1) / BN, per = ksa_div(n_tiles + a.n_splits - 1, a.by_splits);
    const int first_tile = split * per, end_tile = min(n_tiles, first_tile + per);

    // the lane's pair
    const int pair = tile.first + min(wave * 32 + r, n_pairs - 1), in_kind = ksa_div(pair, a.by_group);
    const RowKind kind = {tile.text, base + in_kind};
    const int hq = hkv * a.group + pair - in_kind * a.group, row = seq.first + row_of(a.rows, kind) - seq.start;
    const Seen seen = seen_of(keys, visible(a.rows, kind));
    const bool w_any = wave * 32 < n_pairs, mine = wave * 32 + r < n_pairs;
    bf16x8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = scaled_q(a.q + row * a.q_row + hq * a.q_head + s * 16 + h * 8, a.q_scale);

    // ---- tiles on their way: where their rows are, then into registers, then as bf16 into LDS -------------------------
    const unsigned char *kb = a.k + hkv * a.head_bytes, *vb = a.v + hkv * a.head_bytes;
    const int f_row = lane / LPR, f_piece = lane % LPR;
    Spot spot;            // of row RW * wave + lane % RW of the tile
    int ke = 0, ve = 0;
    u32x4 kr[NI], vr[NI];
    auto look = [&](int t) { spot = spot_of(a.rows, tile.b, key_at(keys, min(t * BN + RW * wave + lane % RW, keys.n - 1))); };
    bool lost = false;
    auto fetch = [&]() {
        const int64_t off = spot_bytes(a, spot);
        lost = spot.page < 0;
        if constexpr (F8) {
            const int64_t at = spot_exp(a, spot, hkv);
            ke = a.k_exp[at], ve = a.v_exp[at];
        }
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int64_t from = lane_value(off, i * RPI + f_row) + f_piece * 16;
            kr[i] = *reinterpret_cast<const u32x4 *>(kb + from), vr[i] = *reinterpret_cast<const u32x4 *>(vb + from);
        }
    };
    auto put = [&](int t, int buf) {
        unsigned char *const to = lds + buf * 2 * BYTES;
        const bool whole = every.sees_all(t * BN, t * BN + BN);
        bool odd = false;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int at = i * RPI + f_row, y = RW * wave + at;
            u32x4 k[F8 ? 2 : 1], v[F8 ? 2 : 1];
            as_bf16<F8>(kr[i], F8 ? power_of_two(__shfl(ke, at)) : 1.f, k);
            as_bf16<F8>(vr[i], F8 ? power_of_two(__shfl(ve, at)) : 1.f, v);
#pragma unroll
            for (int z = 0; z < (F8 ? 2 : 1); ++z) {
                const int piece = f_piece * (F8 ? 2 : 1) + z;
                if (!whole) odd |= take_out(v[z]);
                *reinterpret_cast<u32x4 *>(to + y * (D * 2) + ((piece ^ k_swz<D>(y)) << 4)) = k[z];
                *reinterpret_cast<u32x4 *>(to + BYTES + y * (D * 2) + ((piece ^ v_swz<D>(y)) << 4)) = v[z];
            }
        }
        const uint64_t none = __builtin_amdgcn_ballot_w64(lost), taken = __builtin_amdgcn_ballot_w64(odd);
        if (lane == 0) {
            reinterpret_cast<uint16_t *>(&sh_lost[buf])[wave] = (uint16_t)none;
            sh_odd[buf][wave] = taken != 0;
        }
    };

    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 16; ++g) o[db][g] = 0.f;
    float m_run = LOWEST, l_run = 0.f;
    const int grp = lane >> 4, li = lane & 15;
    const int t_row = 4 * (grp >> 1) + (li >> 2), t_col = 16 * (grp & 1) + 4 * (li & 3);
    const int ll_k = r * (D * 2) + ((k_swz<D>(r) ^ h) << 4);
    const int ll_v = BYTES + t_row * (D * 2) + (((t_col >> 3) ^ v_swz<D>(t_row)) << 4) + ((t_col & 7) << 1);

    if (first_tile < end_tile) {
        look(first_tile);
        fetch();
        look(first_tile + 1);
        put(first_tile, 0);
        fetch();
        look(first_tile + 2);
    }
    __syncthreads();
    for (int t = first_tile; t < end_tile; ++t) {
        const int buf = (t - first_tile) & 1, x0 = t * BN;
        const unsigned char *const at = lds + buf * 2 * BYTES;
        const uint64_t none = sh_lost[buf];
        if (w_any && __builtin_amdgcn_ballot_w64(seen.sees_any(x0, x0 + BN)) != 0) {
            f32x16 s[2];
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int g = 0; g < 16; ++g) s[y][g] = 0.f;
#pragma unroll
            for (int x = 0; x < KS; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    s[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(at + ((ll_k ^ (x << 5)) + y * 32 * (D * 2))), q[x], s[y], 0, 0, 0);
            const bool whole = none == 0 && __builtin_amdgcn_ballot_w64(!seen.sees_all(x0, x0 + BN)) == 0;
            float mx = LOWEST;
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int g = 0; g < 16; ++g) s[y][g] *= a.score_scale;
            if (!whole) {
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int g = 0; g < 16; ++g) {
                        const int key = y * 32 + 8 * (g / 4) + 4 * h + g % 4;
                        s[y][g] = !seen.sees(x0 + key) ? -INFINITY : (none >> key) & 1 ? __builtin_nanf("") : s[y][g];
                    }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int g = 0; g < 16; ++g) mx = fmaxf(mx, s[y][g]);
            if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
                mx = fmaxf(fmaxf(mx, swap32(mx)), m_run);
                const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
                m_run = mx, l_run *= alpha;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int g = 0; g < 16; ++g) o[db][g] *= alpha;
            }
            bf16x8 p[4];
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int g = 0; g < 16; ++g) {
                    const float w = __builtin_amdgcn_exp2f(s[y][g] - m_run);
                    l_run += w;
                    p[2 * y + g / 8][g % 8] = (__bf16)w;
                }
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const unsigned char *from = at + y * 16 * (D * 2) + (ll_v ^ (db << 6));
                    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(from));
                    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(from + 8 * (D * 2)));
                    const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[y], o[db], 0, 0, 0);
                }
            if ((sh_odd[buf][0] | sh_odd[buf][1] | sh_odd[buf][2] | sh_odd[buf][3]) != 0) {
                for (int key = 0; key < BN; ++key) {
                    const Spot sp = spot_of(a.rows, tile.b, key_at(keys, min(x0 + key, keys.n - 1)));
                    const bool see = seen.sees(x0 + key);
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            float y[4];
                            no_numbers<F8>(a, hkv, sp, db * 32 + 8 * g + 4 * h, y);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[db][4 * g + e] += see ? y[e] : 0.f;
                        }
                }
            }
        }
        if (t + 1 < end_tile) {
            put(t + 1, buf ^ 1);
            fetch();
            look(t + 3);
        }
        __syncthreads();
    }

    // ---- results ---------------------------------------------------------------------------------------------------------
    const float l = l_run + swap32(l_run);
    if (!mine) return;
    if (a.n_splits == 1) {
        __bf16 *to = a.o + row * a.o_row + hq * a.o_head;
        const float inv = 1.f / l;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                bf16x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[db][4 * g + e] * inv);
                *reinterpret_cast<bf16x4 *>(to + db * 32 + 8 * g + 4 * h) = y;
            }
        if (a.lse && h == 0) a.lse[(int64_t)row * a.n_q_heads + hq] = log_sum(m_run, l);
    } else {
        float *rec = a.ws + (((int64_t)row * a.n_q_heads + hq) * a.n_splits + split) * (D + 4);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4 *>(rec + db * 32 + 8 * g + 4 * h) = f32x4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
        if (h == 0) rec[D] = m_run, rec[D + 1] = l;
    }
}

// ---- the spans' records of one (row, query head) joined, one wave each ------------------------------------------------------

template <int D>
__global__ __launch_bounds__(256) void ksa_paged_join_kernel(const FwdArgs a) {
    constexpr int EACH = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t x = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = (int)(x / a.n_q_heads), hq = (int)(x - (int64_t)row * a.n_q_heads);
    if (row >= a.rows.total) return;
    const int b = sequence_of(a.rows, row);
    if (b == a.rows.batch) return;
    const NewRows seq = new_rows(a.rows, b, a.max_rows);
    if (row < seq.first || row >= seq.first + seq.n) return;
    float out[EACH], M = LOWEST, den = 0.f;
#pragma unroll
    for (int e = 0; e < EACH; ++e) out[e] = __builtin_nanf("");
    if (seq.ok) {
#pragma unroll
        for (int e = 0; e < EACH; ++e) out[e] = 0.f;
        const float *rec = a.ws + x * a.n_splits * (D + 4);
        for (int s = lane; s < a.n_splits; s += 64) M = fmaxf(M, rec[(int64_t)s * (D + 4) + D]);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
        for (int s = 0; s < a.n_splits; ++s) {
            const float *at = rec + (int64_t)s * (D + 4);
            const float w = __builtin_amdgcn_exp2f(at[D] - M);
            den += at[D + 1] * w;
#pragma unroll
            for (int e = 0; e < EACH; ++e) out[e] += at[lane * EACH + e] * w;
        }
    } else {
        den = __builtin_nanf("");
    }
    __bf16 *to = a.o + row * a.o_row + hq * a.o_head + lane * EACH;
#pragma unroll
    for (int e = 0; e < EACH; ++e) to[e] = (__bf16)(out[e] / den);
    if (a.lse && lane == 0) a.lse[x] = log_sum(M, den);
}

template <int D, bool F8>
void launch(const FwdArgs &a, const KsaPagedPlan &plan, hipStream_t st) {
    const dim3 few(plan.n_splits, a.n_kv_heads, a.rows.batch);
    if (plan.columns == 16) hipLaunchKernelGGL((ksa_paged_few_kernel<D, F8, 16>), few, dim3(FEW_WAVES * 64), 0, st, a);
    else if (plan.columns == 32) hipLaunchKernelGGL((ksa_paged_few_kernel<D, F8, 32>), few, dim3(FEW_WAVES * 64), 0, st, a);
    else hipLaunchKernelGGL((ksa_paged_many_kernel<D, F8>), dim3((unsigned)(plan.slots * plan.n_splits * a.n_kv_heads)), dim3(NW * 64), 0, st, a);
    if (plan.n_splits > 1)
        hipLaunchKernelGGL((ksa_paged_join_kernel<D>), dim3((unsigned)(((int64_t)a.rows.total * a.n_q_heads + 3) / 4)), dim3(256), 0, st, a);
}

}  // namespace

int ksa_launch_paged_fwd(const KsaPagedFwd &L, void *stream) {
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
    a.by_group = ksa_divisor(a.group), a.by_heads = ksa_divisor(a.n_kv_heads), a.by_splits = ksa_divisor(a.n_splits);
    // With the first factor in q the products are no larger than the scaled scores and at least half as large, so that they do not
    // overflow where those would not.
    const float scale = p.softmax_scale * 1.4426950408889634f;
    int exponent = 0;
    (void)std::frexp(scale, &exponent);
    a.q_scale = std::ldexp(1.f, std::max(std::min(exponent - 1, 0), -8)), a.score_scale = scale / a.q_scale;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool f8 = L.call.cache.format == KSA_CACHE_FP8;
    if (p.head_dim == 128) f8 ? launch<128, true>(a, L.plan, st) : launch<128, false>(a, L.plan, st);
    else f8 ? launch<64, true>(a, L.plan, st) : launch<64, false>(a, L.plan, st);
    return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP;
}
