// Rotary positions of whole augmented sequences, there and back, and of one row of each.  Data movement, bound by HBM: a wave has a row, or a part of its heads; its lanes work out
// the row's cosines and sines, one pair each, share them in LDS and then go over the heads, 16 bytes of one per lane and the 16 that they are paired with (from the
// cache: the same lines).  36864 rows, 40 heads of 128, 755 MB: 130 us, 5.8 TB/s (a copy on this card 5.0); 12022 rows, 16 heads of 64 11.3 us, 4.9; 100 rows 3; single rows of 64, 512 and
// 4096 sequences 2.9, 4.6 and 15.2.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ksa_rotary.h"

namespace {

struct Args {
    RotaryArgs rotary;
    const __bf16 *in[2];
    __bf16 *out[2];
    int64_t in_batch[2], in_row[2], in_head[2], out_batch[2], out_row[2], out_head[2];
    int32_t heads[2];
    int32_t rows, units, parts;   // rows of a sequence; rows of all times parts
    int32_t c;
    float sign;
    KsaDivisor by_parts, by_rows, by_w;
    int32_t w;
    const int32_t *pos;           // [batch]; one row of each sequence
    int32_t per_position, most;   // summaries of a chunk (0: text indices); what is from `most` on is outside
    KsaDivisor by_position;
};

// Outputs of this many bytes and more, which the caches (256 MB behind the L2s) cannot keep as a whole for whoever reads them next, go past them.  Kept and past (us), 40 heads
// of 128: the call alone with 264 MB of outputs 102 and 86, 378 MB 141 and 136, 1 GB 387 and 380; there and back 378 MB 272 and 261.  Who reads them next pays for a part of that: the
// call and an elementwise pass over its outputs 264 MB 195 and 205, 378 MB 273 and 286, 1 GB 730 and 745; the call and the prefill (64-row chunks) 264 MB 754 and 758, 378 MB 1386 and
// 1395, 512 MB 2289 and 2279, 1 GB 7841 and 7806.  Below the line the next kernel finds more there than going past saves: 96 MB alone 32.8 and 32.6, with the pass 67 and
// 72, with the prefill 159 and 170; 224 MB 87 and 70, 167 and 174, 576 and 584.
constexpr int64_t PAST_CACHES = (int64_t)256 << 20;

template <int D, int P, bool PAST>
__global__ __launch_bounds__(256) void ksa_rotary_kernel(const Args a) {
    constexpr int LANES = D / 8, PER = 64 / LANES, AT_ONCE = 4;   // lanes of a head, heads of a wave's access, accesses on their way
    __shared__ __align__(16) float table[4][64][2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int unit = (int)blockIdx.x * 4 + wave;
    if (unit >= a.units) return;
    const int row = ksa_div(unit, a.by_parts), part = unit - row * a.parts, b = ksa_div(row, a.by_rows), at = row - b * a.rows;
    const int piece = lane % LANES;
    const int all = a.heads[0] + a.heads[1], step = PER * a.parts;
    int position;
    if (a.pos) {
        const int p = a.pos[b];
        if ((unsigned)p >= (unsigned)a.most) {
            for (int h = part * PER + lane / LANES; h < all; h += step) {
                const int of = h >= a.heads[0] ? 1 : 0, head = h - (of ? a.heads[0] : 0);
                __bf16 *const to = of ? a.out[1] + b * a.out_batch[1] + head * a.out_head[1] : a.out[0] + b * a.out_batch[0] + head * a.out_head[0];
                *reinterpret_cast<u32x4 *>(to + piece * 8) = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};   // NaN
            }
            return;
        }
        position = a.per_position ? ksa_div(p, a.by_position) * a.c + a.c - 1 : p;   // (a summary's: the last text of its chunk)
    } else {
        const int j = ksa_div(at, a.by_w);
        position = j * a.c + min(at - j * a.w, a.c - 1);
    }
    const Turn t = turn_at<P>(a.rotary, position, a.sign, piece, table[wave]);
    for (int h0 = part * PER + lane / LANES; h0 < all; h0 += step * AT_ONCE) {
        Piece<P> x[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int h = min(h0 + i * step, all - 1), of = h >= a.heads[0] ? 1 : 0, head = h - (of ? a.heads[0] : 0);
            const __bf16 *const from = of ? a.in[1] + b * a.in_batch[1] + at * a.in_row[1] + head * a.in_head[1] : a.in[0] + b * a.in_batch[0] + at * a.in_row[0] + head * a.in_head[0];
            x[i] = load_piece<P>(a.rotary, from, piece);
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int h = h0 + i * step, of = h >= a.heads[0] ? 1 : 0, head = h - (of ? a.heads[0] : 0);
            if (h >= all) break;
            __bf16 *const to = of ? a.out[1] + b * a.out_batch[1] + at * a.out_row[1] + head * a.out_head[1] : a.out[0] + b * a.out_batch[0] + at * a.out_row[0] + head * a.out_head[0];
            u32x4 *const at_piece = reinterpret_cast<u32x4 *>(to + piece * 8);
            const u32x4 y = turned<P>(a.rotary, x[i], piece, t);
            if constexpr (PAST) __builtin_nontemporal_store(y, at_piece);
            else *at_piece = y;
        }
    }
}

template <int D, int P>
void launch(const Args &a, hipStream_t st) {
    const dim3 grid((unsigned)((a.units + 3) / 4));
    if ((int64_t)a.units / a.parts * (a.heads[0] + a.heads[1]) * D * 2 >= PAST_CACHES) hipLaunchKernelGGL((ksa_rotary_kernel<D, P, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((ksa_rotary_kernel<D, P, false>), grid, dim3(256), 0, st, a);
}
template <int D>
void launch(const Args &a, int pairs, hipStream_t st) {
    if (pairs == KSA_HALF) launch<D, KSA_HALF>(a, st);
    else if (pairs == KSA_NEXT) launch<D, KSA_NEXT>(a, st);
    else launch<D, KSA_HALF_ANY>(a, st);
}

}  // namespace

int ksa_launch_rotary(const KsaRotaryCall &L, void *stream) {
    Args a;
    a.rotary = {L.rotary.turns, L.rotary.dim, L.rotary.magnitude};
    for (int x = 0; x < 2; ++x) {
        a.in[x] = static_cast<const __bf16 *>(L.in[x]), a.out[x] = static_cast<__bf16 *>(L.out[x]);
        a.in_batch[x] = L.in_strides[x][0], a.in_row[x] = L.in_strides[x][1], a.in_head[x] = L.in_strides[x][2];
        a.out_batch[x] = L.out_strides[x][0], a.out_row[x] = L.out_strides[x][1], a.out_head[x] = L.out_strides[x][2];
    }
    a.heads[0] = L.in[0] ? L.p.n_q_heads : 0, a.heads[1] = L.in[1] ? L.p.n_kv_heads : 0;
    a.rows = L.rows;
    const int rows = L.rows * L.p.batch, accesses = ((a.heads[0] + a.heads[1]) * L.p.head_dim + 511) / 512;
    // Few rows: a row's heads are dealt to several waves, up to 4096 of them. Two calls, with 1024, 4096 and 16384 (us): 112 rows 5.9, 6.2, 6.2; 450 rows 8.4, 9.0, 9.3;
    // 1700 rows 18.9, 17.7, 22.5; 3400 rows 28.0, 27.9, 26.6.
    a.parts = std::max(1, std::min(accesses, 4096 / rows));
    a.units = rows * a.parts;
    a.c = L.p.chunk_len, a.w = a.c + (L.p.chunk_len > L.p.n_text ? 0 : L.p.n_summary);   // (a chunk that is never whole has no summaries)
    a.sign = L.back ? -1.f : 1.f;
    a.pos = L.pos, a.per_position = L.kind == KSA_ROW_SUMMARY ? L.p.n_summary : 0;
    a.most = L.kind == KSA_ROW_SUMMARY ? L.p.n_text / L.p.chunk_len * L.p.n_summary : L.p.n_text;
    a.by_position = ksa_divisor(std::max(a.per_position, 1));
    a.by_parts = ksa_divisor(a.parts), a.by_rows = ksa_divisor(a.rows), a.by_w = ksa_divisor(a.w);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (L.p.head_dim == 128) launch<128>(a, rotary_pairs(L.rotary), st);
    else launch<64>(a, rotary_pairs(L.rotary), st);
    return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP;
}
