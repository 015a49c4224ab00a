// Rotary positions: what the argument checks hand to the kernels, and the turn itself.
#ifndef KSA_ROTARY_H_
#define KSA_ROTARY_H_

#include <stdint.h>

#include "ksa.h"

// Whole sequences, or (pos) one row of each: q, k and their outputs, any of the pairs null.  Strides {batch, row, head} in elements.
struct KsaRotaryCall {
    ksa_params p;
    ksa_rotary rotary;
    int32_t rows;                 // of a sequence
    bool back;                    // turned back
    const int32_t *pos;           // the rows' text indices, or summary ordinals
    int32_t kind;                 // KSA_ROW_*
    const void *in[2];            // q, k
    void *out[2];
    int64_t in_strides[2][3], out_strides[2][3];
};
int ksa_launch_rotary(const KsaRotaryCall &a, void *stream);

// INVALID_ARG if something about it makes no sense
inline int ksa_check_rotary(const ksa_rotary *r, int32_t head_dim) {
    if (!r || r->dim < 2 || r->dim > head_dim || r->dim % 2 != 0 || (r->interleaved != 0 && r->interleaved != 1) || r->reserved != 0) return KSA_ERR_INVALID_ARG;
    if (!(r->magnitude > 0.f) || r->magnitude > 3.402823e38f || !r->turns || reinterpret_cast<uintptr_t>(r->turns) % 8 != 0) return KSA_ERR_INVALID_ARG;
    return KSA_OK;
}

#ifdef __HIPCC__
#include "ksa_device.h"

namespace {

struct RotaryArgs {
    const uint64_t *turns;
    int32_t dim;
    float magnitude;
};

// Which element a piece's elements are paired with: KSA_HALF, KSA_HALF_ANY: dim / 2 further or back (KSA_HALF: dim is a multiple of 16, so that a piece of 8 elements
// is paired with a whole one); KSA_NEXT: the neighbour.
enum { KSA_HALF, KSA_HALF_ANY, KSA_NEXT };
inline int rotary_pairs(const ksa_rotary &r) { return r.interleaved ? KSA_NEXT : r.dim % 16 == 0 ? KSA_HALF : KSA_HALF_ANY; }

// cos and sin of a position times a frequency.  The product is taken modulo a turn in 64 bits of fixed point, its first 32 bits are kept; by
// the quarter turn nearest to it what is left is at most pi / 4, where Taylor's series up to x^9 and x^8 are off by 2e-9 and 2.5e-8.
// Both are within 2^-22.
__device__ __forceinline__ void turn_of(uint64_t turns, int position, float &c, float &s) {
    const unsigned u = (unsigned)((turns * (uint64_t)(unsigned)position) >> 32), quarter = (u + (1u << 29)) >> 30;
    const float x = (float)(int)(u - (quarter << 30)) * 1.4629180792671596e-9f, x2 = x * x;   // 2 pi / 2^32
    const float sine = x + x * x2 * fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6);
    const float cosine = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 40320, -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const float a = quarter & 1 ? sine : cosine, b = quarter & 1 ? cosine : sine;
    c = (quarter + 1) & 2 ? -a : a, s = quarter & 2 ? -b : b;
}

// The turns of the 8 elements of piece `piece` of a head, by position: element e becomes c[e] x + s[e] (its partner).  `table` is memory of the wave's own, 64 pairs.
struct Turn {
    float c[8], s[8];
};
template <int P>
__device__ __forceinline__ Turn turn_at(const RotaryArgs &a, int position, float sign, int piece, float (*table)[2]) {
    const int lane = threadIdx.x & 63, pairs = a.dim / 2;
    if (lane < pairs) {
        float c, s;
        turn_of(a.turns[lane], position, c, s);
        table[lane][0] = c * a.magnitude, table[lane][1] = s * (sign * a.magnitude);
    }
    __builtin_amdgcn_wave_barrier();   // (a wave's LDS accesses are carried out in order)
    Turn t;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int i = piece * 8 + e, pair = P == KSA_NEXT ? i / 2 : i >= pairs ? i - pairs : i;
        const bool second = P == KSA_NEXT ? e & 1 : i >= pairs;
        const int at = min(pair, pairs - 1);   // (elements from dim on are not turned)
        t.c[e] = table[at][0], t.s[e] = second ? table[at][1] : -table[at][1];
    }
    return t;
}

// A piece and what it is paired with, as they lie in memory; then turned.
template <int P>
struct Piece {
    u32x4 own, other;
};
template <int P>
__device__ __forceinline__ Piece<P> load_piece(const RotaryArgs &a, const __bf16 *head, int piece) {
    Piece<P> x;
    x.own = *reinterpret_cast<const u32x4 *>(head + piece * 8);
    if constexpr (P == KSA_HALF) {
        const int i = piece * 8, half = a.dim / 2;
        x.other = *reinterpret_cast<const u32x4 *>(head + (i < half ? i + half : i < a.dim ? i - half : i));
    } else if constexpr (P == KSA_HALF_ANY) {
        const int half = a.dim / 2;
        const unsigned short *const from = reinterpret_cast<const unsigned short *>(head);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            unsigned y = 0;
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                const int i = piece * 8 + 2 * e + z;
                y |= (unsigned)from[i < half ? i + half : i < a.dim ? i - half : i] << (16 * z);
            }
            x.other[e] = y;
        }
    }
    return x;
}
template <int P>
__device__ __forceinline__ u32x4 turned(const RotaryArgs &a, const Piece<P> &x, int piece, const Turn &t) {
    u32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float lo = __builtin_bit_cast(float, x.own[e] << 16), hi = __builtin_bit_cast(float, x.own[e] & 0xffff0000u);
        float lo_of = hi, hi_of = lo;
        if constexpr (P != KSA_NEXT) lo_of = __builtin_bit_cast(float, x.other[e] << 16), hi_of = __builtin_bit_cast(float, x.other[e] & 0xffff0000u);
        const __bf16 z[2] = {(__bf16)fmaf(lo, t.c[2 * e], lo_of * t.s[2 * e]), (__bf16)fmaf(hi, t.c[2 * e + 1], hi_of * t.s[2 * e + 1])};
        const unsigned z0 = __builtin_bit_cast(unsigned short, z[0]), z1 = __builtin_bit_cast(unsigned short, z[1]);
        const int i = piece * 8 + 2 * e;
        // (what is not turned keeps its bits; KSA_HALF_ANY, and KSA_NEXT where dim is no multiple of 8, have pieces of both)
        y[e] = (i < a.dim ? z0 : x.own[e] & 0xffffu) | (i + 1 < a.dim ? z1 << 16 : x.own[e] & 0xffff0000u);
    }
    return y;
}

}  // namespace
#endif

#endif
