// Attention over a paged cache of 4-bit rows.
#include "ksa_paged_fwd.h"

namespace {

// Few rows.  As ksa_paged_few_kernel: every wave streams blocks of 32 keys of its own, once for all pairs, with the running maximum and sum of a softmax.  A row
// is a quarter of a bf16 one, so what is done per key counts for more than there:
//   - A lane loads a row's pieces where the first product wants them: the order of a product's columns is free, so a lane's 16 bytes, a group of 32 elements with one
//     exponent, are its operands of four products one after the other.  K goes through the conversion to bf16 (exact) but not through LDS.
//   - With at most 16 pairs the products have 16 columns: half the weights, half the products' time and half the accumulators of 32.
//   - V is converted where it was loaded, goes through LDS as bf16 and comes back transposed; K's rows are V's, so that an entry is looked up once.
// 64 sequences at 128K, 32/8 heads, 1.15 GB: 170 us, 6.7 TB/s (through the kernel of the other formats 277), of the 6.5 - 6.8 that a plain read reaches; the
// vector unit issues 72 % of the time, 227 instructions per block. 16 sequences of 1 .. 8 rows, 32 columns, 100 MB: 34 us in four spans; there the matrix unit's time and the vector
// instructions' (237 per block) add up to 90 % of it. One of 700 keys 4.9 us. Dropped (us, before and after): one scalar address for keys side by side in a page
// (128K 198, 206), two blocks on their way (16 columns have no registers for them: 181, 315; 32 columns level), operands of V read ahead of the weights (level), 64 keys
// per block for 32 columns (32 x 8 rows at 128K 124, 121; the 16 sequences 34.8, 36), two workgroups of 16 columns for 32 pairs (127, 176), loads that stay in the
// caches (128K 182, 200). Products of 4-bit K with q in two 8-bit parts, which need no conversion, are exact one by one, but the matrix unit's sums of them are not: off by
// 2^-18 of the terms' sizes, by 2^-13 where q's elements are 2^10 apart.
template <int COLS>
struct Acc;
template <>
struct Acc<16> {
    typedef f32x4 type;
};
template <>
struct Acc<32> {
    typedef f32x16 type;
};
template <int COLS, class T>
__device__ __forceinline__ T product(const bf16x8 &a, const bf16x8 &b, const T &c) {
    if constexpr (COLS == 16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// The value of the lane 16 away (32: of the lane 32 away) in the other half of each 32 (64).
__device__ __forceinline__ float other_quarter(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __builtin_bit_cast(float, (threadIdx.x & 16) ? r[0] : r[1]);
}
template <int COLS>
__device__ __forceinline__ float most_of_column(float x) {
    x = fmaxf(x, other_half(x));
    return COLS == 16 ? fmaxf(x, other_quarter(x)) : x;
}
template <int COLS>
__device__ __forceinline__ float sum_of_column(float x) {
    x += other_half(x);
    return COLS == 16 ? x + other_quarter(x) : x;
}

// A row's reference is raised only where a score exceeds it by this many powers of two: a weight is at most 8, and after the first blocks the outputs are hardly ever scaled
// (32 columns: of the 70 % of all blocks in which some column's largest score grows none is left; 32 sequences of 8 rows at 128K 126.6 us -> 123.4).
constexpr float SLACK = 3.f;

template <int D, int COLS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, COLS == 16 || D == 64 ? 4 : 2) void ksa_paged_few_fp4_kernel(const FwdArgs a) {
    typedef typename Acc<COLS>::type acc;
    constexpr int GROUPS = 64 / COLS;                   // of lanes with the same pair
    constexpr int ROWS = BLOCK / COLS;                  // of a block, per lane
    constexpr int BYTES = D / 2 / GROUPS;               // of a row, per lane: 8, 16 or 32
    constexpr int WORDS = BYTES / 4, PIECES = BYTES / 16 < 1 ? 1 : BYTES / 16, EACH = WORDS / PIECES;   // pieces of EACH words of one group
    constexpr int KS = WORDS, TILES = ROWS;             // products per tile of COLS keys, tiles of a block
    constexpr int AB = D / COLS, PER = COLS == 16 ? 4 : 16;   // blocks of columns of the output, values of a product per lane
    constexpr int VROW = D * 2 + 48;                    // bytes: conflicts are 25 % of the LDS cycles of 32 columns, with 32 more bytes 49 %, with 64 66 %
    constexpr int OWN = BLOCK * VROW, PARTS = COLS / 16, PART = D / PARTS, OUT_ROW = PART + 4;   // the results pass through the blocks' memory, in parts of the columns
    static_assert(COLS * OUT_ROW * 4 <= OWN, "a part of a wave's results lies where its blocks were");
    __shared__ __align__(16) unsigned char lds[WAVES * OWN];
    __shared__ float sh_m[WAVES][COLS], sh_l[WAVES][COLS];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane % COLS, g = lane / COLS;
    const int split = blockIdx.x, hkv = blockIdx.y, b = blockIdx.z;
    const NewRows seq = new_rows(a.rows, b, a.max_rows);
    if (seq.n == 0) return;
    if (!seq.ok) {
        if (a.n_splits > 1) return;   // (the joining kernel sees to it)
        for (int x = tid / D; x < seq.n * a.group; x += WAVES * 64 / D) {
            const int row = x / a.group, hq = hkv * a.group + x % a.group;
            a.o[(seq.first + row) * a.o_row + hq * a.o_head + tid % D] = (__bf16)__builtin_nanf("");
            if (a.lse && tid % D == 0) a.lse[(int64_t)(seq.first + row) * a.n_q_heads + hq] = __builtin_nanf("");
        }
        return;
    }
    const Keys keys = keys_of(a.rows, seq.start, seq.start + seq.n - 1);
    const int per = ksa_div((keys.n + BLOCK - 1) / BLOCK + a.n_splits - 1, a.by_splits) * BLOCK;
    const int v0 = split * per, v1 = min(keys.n, v0 + per);

    // ---- blocks on their way: table entries two ahead, rows one ahead.  Lane: rows r, r + COLS, .. of a block; of each the bytes from 16 g on, and 16 GROUPS further
    // (8 g where a row has 32 bytes for four lanes). ---------------------------------------------------------------------------------
    typedef unsigned piece_t __attribute__((ext_vector_type(EACH)));
    const unsigned char *const kb = a.k + hkv * a.head_bytes, *const vb = a.v + hkv * a.head_bytes;
    const uint8_t *const k_exp = a.k_exp + ((int64_t)hkv << a.rows.shift) * (D / 32), *const v_exp = a.v_exp + ((int64_t)hkv << a.rows.shift) * (D / 32);
    const unsigned exp_page = ((unsigned)a.n_kv_heads << a.rows.shift) * (D / 32);   // exponents of a page
    auto byte_of = [&](int z) { return (z * GROUPS + g) * EACH * 4; };   // of a row: the lane's piece z
    struct {
        piece_t k[ROWS][PIECES], v[ROWS][PIECES];
        int ke[ROWS][PIECES], ve[ROWS][PIECES];
        unsigned lost;         // keys without a page
    } next;                    // the one on its way
    Entry entry[ROWS];         // of the block to be requested next
    auto look = [&](int x) {
#pragma unroll
        for (int y = 0; y < ROWS; ++y) entry[y] = entry_of(a.rows, b, key_at(keys, min(x + y * COLS + r, keys.n - 1)));
    };
    auto request = [&](int x_next) {
        unsigned page[ROWS], slot[ROWS];
        next.lost = 0;
#pragma unroll
        for (int y = 0; y < ROWS; ++y) {
            const Spot spot = spot_of(a.rows, entry[y]);
            const unsigned none = (unsigned)__builtin_amdgcn_ballot_w64(spot.page < 0);
            next.lost |= COLS == 16 ? (none & 0xffffu) << (16 * y) : none;
            page[y] = max(spot.page, 0), slot[y] = spot.slot;
        }
        look(x_next);   // (loads return in the order they are issued in)
#pragma unroll
        for (int y = 0; y < ROWS; ++y) {
            const uint64_t at = (uint64_t)page[y] * exp_page + (slot[y] * (D / 32) + byte_of(0) / 16);
#pragma unroll
            for (int z = 0; z < PIECES; ++z) next.ke[y][z] = k_exp[at + z * GROUPS], next.ve[y][z] = v_exp[at + z * GROUPS];
        }
        uint64_t at[ROWS];     // (strides fit 32 bits)
#pragma unroll
        for (int y = 0; y < ROWS; ++y) at[y] = (uint64_t)page[y] * (unsigned)a.page_bytes + slot[y] * (unsigned)a.row_bytes + byte_of(0);
#pragma unroll
        for (int y = 0; y < ROWS; ++y)
#pragma unroll
            for (int z = 0; z < PIECES; ++z) next.k[y][z] = __builtin_nontemporal_load(reinterpret_cast<const piece_t *>(kb + at[y] + z * GROUPS * 16));
#pragma unroll
        for (int y = 0; y < ROWS; ++y)
#pragma unroll
            for (int z = 0; z < PIECES; ++z) next.v[y][z] = __builtin_nontemporal_load(reinterpret_cast<const piece_t *>(vb + at[y] + z * GROUPS * 16));
    };
    constexpr int STEP = WAVES * BLOCK;
    const int first = v0 + wave * BLOCK;
    if (first < v1) {
        look(first);
        request(first + STEP);
    }

    // the lane's pair = row * group + head (the last one repeats)
    const int pairs = seq.n * a.group, pair = min(r, pairs - 1), q_row = ksa_div(pair, a.by_group), q_head = hkv * a.group + pair - q_row * a.group;
    const Seen seen = seen_of(keys, visible(a.rows, kind_of(a.rows, seq.start + q_row)));
    bf16x8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s)
        q[s] = scaled_q(a.q + (seq.first + q_row) * a.q_row + q_head * a.q_head + byte_of(s / EACH) * 2 + s % EACH * 8, a.q_scale);

    acc o[AB];
    float m_run = LOWEST, l_run = 0.f;
#pragma unroll
    for (int x = 0; x < AB; ++x)
#pragma unroll
        for (int i = 0; i < PER; ++i) o[x][i] = 0.f;
    unsigned char *const own = lds + wave * OWN;
    unsigned char *const put_at = own + r * VROW;
    // Transposing reads: 16 lanes bring 4 keys by 16 columns.  A lane's operand is keys 4 g .. and 16 + 4 g .. (32 columns of pairs: 8 further), of which it has the weights.
    const int grp = lane >> 4, li = lane & 15;
    const unsigned char *const v_at = COLS == 16 ? own + (4 * grp + (li >> 2)) * VROW + 8 * (li & 3) : own + (4 * (grp >> 1) + (li >> 2)) * VROW + 32 * (grp & 1) + 8 * (li & 3);
    constexpr int NEXT = (COLS == 16 ? 16 : 8) * VROW;
    auto sees_all = [&](int x) { return __builtin_amdgcn_ballot_w64(!seen.sees_all(x, x + BLOCK)) == 0; };
    bool ever = false;         // groups of V were taken out
    for (int x = first; x < v1; x += STEP) {
        const unsigned none = next.lost;
        const bool whole = none == 0 && sees_all(x);
        if (!whole) {
            bool odd = false;
#pragma unroll
            for (int y = 0; y < ROWS; ++y)
#pragma unroll
                for (int z = 0; z < PIECES; ++z) {
                    const bool gone = next.ve[y][z] == NO_NUMBERS;
#pragma unroll
                    for (int e = 0; e < EACH; ++e) next.v[y][z][e] = gone ? 0u : next.v[y][z][e];
                    next.ve[y][z] = min(next.ve[y][z], MOST_EXP4), odd |= gone;
                }
            ever |= __builtin_amdgcn_ballot_w64(odd) != 0;
        }
        acc sc[TILES];
#pragma unroll
        for (int y = 0; y < TILES; ++y) {
#pragma unroll
            for (int i = 0; i < PER; ++i) sc[y][i] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s)
                sc[y] = product<COLS>(__builtin_bit_cast(bf16x8, unpack_fp4(next.k[y][s / EACH][s % EACH], power_of_two(next.ke[y][s / EACH]))), q[s], sc[y]);
        }
#pragma unroll
        for (int y = 0; y < ROWS; ++y)
#pragma unroll
            for (int z = 0; z < PIECES; ++z)
#pragma unroll
                for (int e = 0; e < EACH; ++e)
                    *reinterpret_cast<u32x4 *>(put_at + y * COLS * VROW + byte_of(z) * 4 + e * 16) = unpack_fp4(next.v[y][z][e], power_of_two(next.ve[y][z]));
        if (x + STEP < v1) request(x + 2 * STEP);

        // The lane's scores, 16 / GROUPS * 2 of them: keys 4 g + i (16 columns: of each tile), or 8 (i / 4) + 4 h + i % 4.
        if (!whole) {
            const unsigned see = seen.sees_32(x) >> (4 * g), gone = none >> (4 * g);
#pragma unroll
            for (int y = 0; y < TILES; ++y)
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const int bit = COLS == 16 ? 16 * y + i : 8 * (i / 4) + i % 4;
                    const float s = (gone >> bit) & 1 ? __builtin_nanf("") : (float)sc[y][i];
                    sc[y][i] = (see >> bit) & 1 ? s : -__builtin_inff();
                }
        }
        float most = sc[0][0];
#pragma unroll
        for (int y = 0; y < TILES; ++y)
#pragma unroll
            for (int i = 0; i < PER; ++i) most = fmaxf(most, sc[y][i]);
        most = most_of_column<COLS>(most) * a.score_scale;
        if (__builtin_amdgcn_ballot_w64(most > m_run + SLACK) != 0) {
            const float m = most > m_run + SLACK ? most : m_run, alpha = __builtin_amdgcn_exp2f(m_run - m);
            m_run = m, l_run *= alpha;
#pragma unroll
            for (int y = 0; y < AB; ++y)
#pragma unroll
                for (int i = 0; i < PER; ++i) o[y][i] *= alpha;
        }
        bf16x8 p[PER * TILES / 8];
#pragma unroll
        for (int y = 0; y < TILES; ++y)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float w = __builtin_amdgcn_exp2f(fmaf(sc[y][i], a.score_scale, -m_run));
                const int at = y * PER + i;
                l_run += w, p[at / 8][at % 8] = (__bf16)w;
            }
#pragma unroll
        for (int z = 0; z < PER * TILES / 8; ++z)
#pragma unroll
            for (int y = 0; y < AB; ++y) {
                const unsigned char *at = v_at + z * 16 * VROW + y * COLS * 2;
                const s16x4 w0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(at));
                const s16x4 w1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(at + NEXT));
                o[y] = product<COLS>(__builtin_bit_cast(bf16x8, __builtin_shufflevector(w0, w1, 0, 1, 2, 3, 4, 5, 6, 7)), p[z], o[y]);
            }
    }
    if (ever) {   // what was taken out of V, to the rows that see it
        for (int x = first; x < v1; x += STEP)
            for (int key = 0; key < min(BLOCK, keys.n - x); ++key) {
                const Spot at = spot_of(a.rows, entry_of(a.rows, b, key_at(keys, x + key)));
                if (sees_all(x) && at.page >= 0) continue;   // (where a page is missing the sum is none anyway)
                const bool see = seen.sees(x + key);
#pragma unroll
                for (int y = 0; y < AB; ++y)
#pragma unroll
                    for (int i = 0; i < PER; i += 4) {
                        float z[4];
                        no_numbers<D, KSA_CACHE_FP4>(a, hkv, at, y * COLS + (COLS == 16 ? 0 : 2 * i) + 4 * g, z);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[y][i + e] += see ? z[e] : 0.f;
                    }
            }
    }

    // ---- the waves' results ------------------------------------------------------------------------------------------
    const float l = sum_of_column<COLS>(l_run);
    if (g == 0) sh_m[wave][r] = m_run, sh_l[wave][r] = l;
    float *const mine = reinterpret_cast<float *>(own);
    constexpr int LANES = PART / 8;   // lanes per pair
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
        if (part > 0) __syncthreads();
#pragma unroll
        for (int y = part * (AB / PARTS); y < (part + 1) * (AB / PARTS); ++y)
#pragma unroll
            for (int i = 0; i < PER; i += 4)
                *reinterpret_cast<f32x4 *>(mine + r * OUT_ROW + (y - part * (AB / PARTS)) * COLS + (COLS == 16 ? 0 : 2 * i) + 4 * g) = f32x4{o[y][i], o[y][i + 1], o[y][i + 2], o[y][i + 3]};
        __syncthreads();
        for (int x = tid / LANES; x < pairs; x += WAVES * 64 / LANES) {
            const int in = tid % LANES * 8, d0 = part * PART + in;
            float M = sh_m[0][x];
#pragma unroll
            for (int y = 1; y < WAVES; ++y) M = fmaxf(M, sh_m[y][x]);
            float den = 0.f, out[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e] = 0.f;
#pragma unroll
            for (int y = 0; y < WAVES; ++y) {
                const float w = __builtin_amdgcn_exp2f(sh_m[y][x] - M);
                const float *from = reinterpret_cast<const float *>(lds + y * OWN) + x * OUT_ROW + in;
                den += sh_l[y][x] * w;
#pragma unroll
                for (int e = 0; e < 8; ++e) out[e] += from[e] * w;
            }
            const int in_seq = ksa_div(x, a.by_group), row = seq.first + in_seq, hq = hkv * a.group + x - in_seq * a.group;
            if (a.n_splits == 1) {
                bf16x8 z;
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = (__bf16)(out[e] / den);
                *reinterpret_cast<bf16x8 *>(a.o + row * a.o_row + hq * a.o_head + d0) = z;
                if (a.lse && d0 == 0) a.lse[(int64_t)row * a.n_q_heads + hq] = log_sum(M, den);
            } else {
                float *rec = a.ws + (((int64_t)row * a.n_q_heads + hq) * a.n_splits + split) * (D + 4);
#pragma unroll
                for (int e = 0; e < 8; e += 4) *reinterpret_cast<f32x4 *>(rec + d0 + e) = f32x4{out[e], out[e + 1], out[e + 2], out[e + 3]};
                if (d0 == 0) rec[D] = M, rec[D + 1] = den;
            }
        }
    }
}

// Of 16 columns: eight waves to a workgroup where there are at most two on a compute unit (512), so that these have as many as they hold; with more of them
// four.  Measured with four and with eight (us): 64 sequences at 128K, 512 workgroups 192 and 181; 8 at 32K, full attention 53.2 and 50.9; one of 700 keys 5.1 and 4.7;
// 128 of 2000 keys, 1024 workgroups 12.2 and 15.3.
template <int D>
void launch(const FwdArgs &a, const KsaPagedPlan &plan, hipStream_t st) {
    const dim3 few(plan.n_splits, a.n_kv_heads, a.rows.batch);
    if (!plan.few) launch_many<D, KSA_CACHE_FP4>(a, plan, st);
    else if (a.max_rows * a.group > 16) hipLaunchKernelGGL((ksa_paged_few_fp4_kernel<D, 32, 4>), few, dim3(256), 0, st, a);
    else if ((int64_t)plan.n_splits * a.n_kv_heads * a.rows.batch > 512) hipLaunchKernelGGL((ksa_paged_few_fp4_kernel<D, 16, 4>), few, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((ksa_paged_few_fp4_kernel<D, 16, 8>), few, dim3(512), 0, st, a);
}

}  // namespace

void ksa_launch_paged_fwd_fp4(const KsaPagedFwd &L, void *stream) {
    const FwdArgs a = fwd_args(L);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (L.call.p.head_dim == 128) launch<128>(a, L.plan, st);
    else launch<64>(a, L.plan, st);
}
