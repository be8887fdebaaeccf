// What the kernels of attention over the paged cache share.
#pragma once

#include "star_common.hpp"
#include "star_internal.hpp"

namespace star {

constexpr float kLn2 = 0.69314718055994531f;
constexpr int kBlockRows = 16;   // query rows of one row-block (a product's columns)
constexpr int kBlockWaves = 4;   // waves of its workgroup, one tile of keys each a step

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// The keys that the rows at positions p0..p1 of one request can see, in tiles:
// nA tiles of first tokens (sinks), then tiles b0.. up to p1's.
struct Tiles {
    int nA, b0, n;
    __device__ int at(int u) const { return u < nA ? u : u - nA + b0; }
};
template <int kTile>
__device__ inline Tiles tiles_of(const AttendArgs& a, int p0, int p1) {
    Tiles t;
    const int lo = a.window && p0 >= a.window ? p0 - a.window + 1 : 0;
    t.b0 = lo / kTile;
    const int s = a.window ? (a.sinks < p1 + 1 ? a.sinks : p1 + 1) : 0;
    const int nA = (s + kTile - 1) / kTile;
    t.nA = nA < t.b0 ? nA : t.b0;
    t.n = p1 < 0 ? 0 : t.nA + p1 / kTile - t.b0 + 1;
    return t;
}

// One request of the call: L cached tokens, the last T of them new, its rows
// of q from row0 on.  A request that breaks a precondition has no rows.
struct Slot {
    int L, T, row0, blocks;   // blocks of kBlockRows rows
    int steps;                // scheduling steps of one block (kBlockWaves tiles each)
};
template <int kTile>
__device__ inline Slot slot_of(const AttendArgs& a, int b, int32_t& bad) {
    Slot s;
    s.L = a.seq_len[b];
    bool ok = s.L >= 0 && s.L <= a.max_pages << a.ps_log2;
    if (a.q_start) {
        const int from = a.q_start[b], to = a.q_start[b + 1];
        s.row0 = from;
        s.T = to - from;
        ok = ok && from >= 0 && to >= from && to <= a.n_rows && s.T <= s.L;
    } else {
        s.row0 = b;
        s.T = 1;                       // an empty request's row is all zeros
    }
    if (!ok) {
        bad |= STAR_DEV_BAD_LEN;
        s.L = s.T = 0;
    }
    s.blocks = (int)(((int64_t)s.T * a.g + kBlockRows - 1) / kBlockRows);
    int n = tiles_of<kTile>(a, s.L - 1, s.L - 1).n;
    if (s.T > 1 && a.window) {          // a block's rows span at most kBlockRows positions
        const int all = (s.L - 1) / kTile + 1;
        n = n + (kBlockRows + kTile - 1) / kTile + 1;
        n = n < all ? n : all;
    }
    s.steps = n > kBlockWaves ? (n + kBlockWaves - 1) / kBlockWaves : 1;
    return s;
}

// A product's result may be read a number of wait states after it is issued (11
// for these shapes).  The compiler counts them within a basic block; where a
// branch came between, it was seen to count the longer of two paths only
// (fp32, 256 wide: the last product was missing from one register in four).
// So results meet 16 wait states before any branch.
__device__ inline void settle(f32x4& x) { asm volatile("s_nop 15" : "+v"(x)); }
// (32 x 32 products: 19)
__device__ inline void settle(f32x16& x) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(x)); }

template <int kDtype>
__device__ inline bool not_finite(uint32_t w) {
    if constexpr (kDtype == STAR_F32)
        return (w & 0x7F800000u) == 0x7F800000u;
    else
        return (w & 0x7F80u) == 0x7F80u || (w & 0x7F800000u) == 0x7F800000u;
}

// the larger magnitudes, value by value (and the signs dropped)
template <int kDtype>
__device__ inline uint32_t larger(uint32_t a, uint32_t w) {
    if constexpr (kDtype == STAR_F32) return max(a, w & 0x7FFFFFFFu);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(
                                            __builtin_bit_cast(u16x2, a),
                                            __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)));
}
// the word with its values that are not finite at 0
template <int kDtype>
__device__ inline uint32_t finite_part(uint32_t w) {
    if constexpr (kDtype == STAR_F32) return not_finite<kDtype>(w) ? 0u : w;
    const uint32_t lo = (w & 0x7F80u) == 0x7F80u ? 0u : w & 0xFFFFu;
    const uint32_t hi = (w & 0x7F800000u) == 0x7F800000u ? 0u : w & 0xFFFF0000u;
    return lo | hi;
}
// n outputs of one row
template <int kDtype, int n>
__device__ inline void store_out(char* to, const float* y) {
#pragma unroll
    for (int i = 0; i < n; i += 4) {
        if constexpr (kDtype == STAR_BF16)
            *(u32x2*)(to + 2 * i) =
                u32x2{pack_bf16x2_rne(y[i], y[i + 1]), pack_bf16x2_rne(y[i + 2], y[i + 3])};
        else
            *(f32x4*)(to + 4 * i) = f32x4{y[i], y[i + 1], y[i + 2], y[i + 3]};
    }
}

}  // namespace star
