// A serving step's new rows: q is turned, k is turned and goes with v into the pages, in one launch.  A wave has a packed row or a part of its heads: it looks the
// row's sequence up, works out the cosines and sines (one pair per lane, shared in LDS), and goes over the query heads, then over the KV heads,
// whose page is looked up once.  Bound by HBM, few rows by latency: 12096 rows, 32 + 8 heads of 128, 198 MB 32 us, 6.1 TB/s; one row of each of 64 sequences 3.8 us
// (the append alone 2.8), a launch, the sequence, the entry and the row one behind the other.  Into bf16, 8-bit and 4-bit pages (one call behind the other on the same rows, us): 64
// sequences' single rows 3.0, 3.3, 3.1; 2048 rows of one 9.7, 10.1, 9.3; 13824 of three 60, 54, 51; 36864 of one 167, 153, 146.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ksa_paged_move.h"
#include "ksa_rotary.h"

namespace {

struct Args {
    MoveArgs move;
    RotaryArgs rotary;
    const __bf16 *q;
    __bf16 *q_out;
    int64_t q_row, q_head, out_row, out_head;
    int32_t n_q_heads;            // 0: no q
    int32_t parts;
    KsaDivisor by_parts;
};

template <int D, int F, int P>
__global__ __launch_bounds__(256) void ksa_paged_rotary_kernel(const Args a) {
    constexpr int LANES = D / 8, PER = 64 / LANES;   // lanes of a head, heads of a wave's access
    __shared__ __align__(16) float table[4][64][2];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int unit = (int)blockIdx.x * 4 + wave, row = ksa_div(unit, a.by_parts), part = unit - row * a.parts;
    const PagedRows &rows = a.move.rows;
    if (row >= rows.total) return;
    int b;
    const NewRows r = sequence_of<1>(rows, row, row, rows.total, b);
    if (row < r.first || row >= r.first + r.n) return;   // a row of no sequence
    const int piece = lane % LANES, step = PER * a.parts, first = part * PER + lane / LANES;
    if (!r.ok) {
        for (int h = first; h < a.n_q_heads; h += step)
            *reinterpret_cast<u32x4 *>(a.q_out + row * a.out_row + h * a.out_head + piece * 8) = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};   // NaN
        return;
    }
    const int aug = r.start + (row - r.first), j = ksa_div(aug, rows.by_w), position = j * rows.c + min(aug - j * (rows.c + rows.m), rows.c - 1);
    const Spot spot = spot_of(rows, entry_of(rows, b, kind_of(rows, aug)));
    const Turn t = turn_at<P>(a.rotary, position, 1.f, piece, table[wave]);
    for (int h = first; h < a.n_q_heads; h += step) {
        const Piece<P> x = load_piece<P>(a.rotary, a.q + row * a.q_row + h * a.q_head, piece);
        *reinterpret_cast<u32x4 *>(a.q_out + row * a.out_row + h * a.out_head + piece * 8) = turned<P>(a.rotary, x, piece, t);
    }
    if (spot.page < 0) return;
    // (the parts that have the fewest query heads come first)
    const int before = (a.n_q_heads + PER - 1) / PER % a.parts, mine = part >= before ? part - before : part - before + a.parts;
    for (int h = mine * PER + lane / LANES; h < a.move.n_kv_heads; h += step) {
        const int64_t from = row * a.move.row_stride + h * a.move.head_stride;
        const Piece<P> x = load_piece<P>(a.rotary, a.move.k + from, piece);
        const u32x4 v = *reinterpret_cast<const u32x4 *>(a.move.v + from + piece * 8);
        put_piece<D, F>(a.move, Place{row, h, spot.page, spot.slot, true}, piece, turned<P>(a.rotary, x, piece, t), v);
    }
}

template <int D, int F>
void launch(const Args &a, int pairs, dim3 grid, hipStream_t st) {
    if (pairs == KSA_HALF) hipLaunchKernelGGL((ksa_paged_rotary_kernel<D, F, KSA_HALF>), grid, dim3(256), 0, st, a);
    else if (pairs == KSA_NEXT) hipLaunchKernelGGL((ksa_paged_rotary_kernel<D, F, KSA_NEXT>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((ksa_paged_rotary_kernel<D, F, KSA_HALF_ANY>), grid, dim3(256), 0, st, a);
}
template <int D>
void launch(const Args &a, int format, int pairs, dim3 grid, hipStream_t st) {
    if (format == KSA_CACHE_FP8) launch<D, KSA_CACHE_FP8>(a, pairs, grid, st);
    else if (format == KSA_CACHE_FP4) launch<D, KSA_CACHE_FP4>(a, pairs, grid, st);
    else launch<D, KSA_CACHE_BF16>(a, pairs, grid, st);
}

}  // namespace

int ksa_launch_paged_rotary(const KsaPagedRotary &L, void *stream) {
    Args a;
    a.move = move_args(L.move);
    a.rotary = {L.rotary.turns, L.rotary.dim, L.rotary.magnitude};
    a.q = static_cast<const __bf16 *>(L.q), a.q_out = static_cast<__bf16 *>(L.q_out);
    a.q_row = L.q_strides[0], a.q_head = L.q_strides[1], a.out_row = L.out_strides[0], a.out_head = L.out_strides[1];
    const ksa_params &p = L.move.call.p;
    a.n_q_heads = L.q ? p.n_q_heads : 0;
    const int rows = a.move.rows.total, per = 512 / p.head_dim, accesses = (a.n_q_heads + per - 1) / per + (p.n_kv_heads + per - 1) / per;
    // Few rows: a row's heads are dealt to several waves, up to 4096 of them. With 1024, 4096 and 16384 (us): 64 rows 3.1 each; 256 rows 4.2, 3.8, 3.8; 1024 rows 7.2, 6.2, 7.4;
    // 4096 rows 17.4, 17.4, 17.9.
    a.parts = std::max(1, std::min(accesses, 4096 / rows));
    a.by_parts = ksa_divisor(a.parts);
    const dim3 grid((unsigned)(((int64_t)rows * a.parts + 3) / 4));
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (p.head_dim == 128) launch<128>(a, L.move.call.cache.format, rotary_pairs(L.rotary), grid, st);
    else launch<64>(a, L.move.call.cache.format, rotary_pairs(L.rotary), grid, st);
    return hipGetLastError() == hipSuccess ? KSA_OK : KSA_ERR_HIP;
}
