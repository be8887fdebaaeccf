// Attention over the paged key-value cache (include/star.h, "attention over
// the cache"): the row-block kernel behind star_attend_decode and short
// star_attend_prompt calls.
#include "attend.hpp"
#include "star_common.hpp"
#include "star_internal.hpp"

namespace star {

namespace {

constexpr int kRows = kBlockRows;
constexpr int kThreads = 256;    // four waves share a block's keys
constexpr int kWaves = kThreads / kWave;
static_assert(kWaves == kBlockWaves, "one tile a wave and step");

template <int kDtype> struct Elem;
template <> struct Elem<STAR_BF16> {
    static constexpr int kBytes = 2, kTile = 32;   // tokens of one tile: a product's K
};
template <> struct Elem<STAR_F32> {
    static constexpr int kBytes = 4, kTile = 16;
};

// maximum / sum over the four lanes l, l ^ 16, l ^ 32, l ^ 48: two register
// swaps between rows of 16 lanes instead of LDS permutes
__device__ inline float quad_max(float v) {
    auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ inline float quad_sum(float v) {
    auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// ---------------------------------------------------------------------------
// One tile's keys and values in registers.
//
// With r = lane % 16 and c = lane / 16, the scores are the product
// S^T [tokens x rows] = K Q^T, whose result gives lane (r, c) the tokens
// 4c..4c+3 of each 16 for row r.  Those are the contraction slots that the
// second product, O^T [d x rows] = V^T P^T, reads from lane (r, c), so the
// probabilities never leave their lane.  V's rows are read whole (16 lanes one
// row) and lane (r, c) holds d = r E .. r E + E - 1 of its tokens: tile i of
// the second product takes element i of every lane.  No LDS in the loop.
// ---------------------------------------------------------------------------
template <int kDtype, int D>
struct Tile {
    static constexpr int kB = Elem<kDtype>::kBytes, kT = Elem<kDtype>::kTile;
    static constexpr int kHalves = kT / 16;
    static constexpr int E = D / 16;                    // d per lane
    static constexpr int kRowV = E * kB;                // bytes of one lane's share of a V row
    static constexpr int kRowsV = 4 * kHalves;          // V rows per lane
    static constexpr int kChunks = D * kB / 64;         // 16-byte loads of one K row per lane
    u32x4 k[kHalves][kChunks];
    uint32_t v[kRowsV][kRowV / 4];
};

// where one 16-token half of a tile lies: its page (checked), or nowhere
struct Half {
    const char* base;     // the page's first byte of this head's keys, at the half's first token
    bool ok;
};

// A lane's share of a V row.  Values that one block alone reads pass the caches
// by, whole lines at a time (128 requests: 379 -> 362 us, 6.0 TB/s; two long
// ones 79 -> 77; where several blocks read them, 76 -> 93); keys take two
// instructions a line, which only the cache joins (the same for them: 364 ->
// 383).
template <int kDtype, int D, bool kOnce>
__device__ inline void load_row(const char* p, uint32_t* to) {
    constexpr int n = Tile<kDtype, D>::kRowV;
    if constexpr (n == 8) {
        const u32x2 x = kOnce ? __builtin_nontemporal_load((const u32x2*)p) : *(const u32x2*)p;
        to[0] = x[0], to[1] = x[1];
    } else {
#pragma unroll
        for (int i = 0; i < n / 16; ++i) {
            const u32x4* at = (const u32x4*)(p + 16 * i);
            const u32x4 x = kOnce ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
            for (int w = 0; w < 4; ++w) to[4 * i + w] = x[w];
        }
    }
}

// the 16-byte pieces of a K row that lane (r, c) contracts: piece i of the
// four lanes c = 0..3 is 64 consecutive bytes
template <int kDtype, int D>
__device__ inline void load_k(const char* row, int c, u32x4* to) {
#pragma unroll
    for (int i = 0; i < Tile<kDtype, D>::kChunks; ++i)
        to[i] = *(const u32x4*)(row + i * 64 + c * 16);
}

// S^T += K Q^T for one 16-token half
template <int kDtype, int D>
__device__ inline f32x4 scores(const u32x4* k, const u32x4* q) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < Tile<kDtype, D>::kChunks; ++i) {
        if constexpr (kDtype == STAR_BF16) {
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[i]),
                                                        __builtin_bit_cast(bf16x8_t, q[i]), s, 0,
                                                        0, 0);
        } else {
#pragma unroll
            for (int x = 0; x < 4; ++x)
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[i][x]),
                                                         __uint_as_float(q[i][x]), s, 0, 0, 0);
        }
    }
    settle(s);
    return s;
}

// O^T += V^T P^T for one tile; p[4 h + x] = lane (r, c)'s token 4c + x of half h.
// bf16: P enters as a bf16 pair hi + lo (2^-16 relative): the products are
// idle behind the loads, and one bf16 would add its 2^-8 to the output's.
template <int kDtype, int D>
__device__ inline void accumulate(const uint32_t (&v)[Tile<kDtype, D>::kRowsV]
                                                     [Tile<kDtype, D>::kRowV / 4],
                                  const float* p, f32x4* o) {
    if constexpr (kDtype == STAR_BF16) {
        u32x4 hi, lo;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            uint32_t h, l;
            split_bf16x2(p[2 * x], p[2 * x + 1], h, l);
            hi[x] = h, lo[x] = l;
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            u32x4 a;
#pragma unroll
            for (int x = 0; x < 4; ++x)     // element i of rows 2x and 2x + 1
                a[x] = __builtin_amdgcn_perm(v[2 * x + 1][i / 2], v[2 * x][i / 2],
                                             i & 1 ? 0x07060302u : 0x05040100u);
            const bf16x8_t va = __builtin_bit_cast(bf16x8_t, a);
            o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8_t, hi),
                                                           o[i], 0, 0, 0);
            o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(bf16x8_t, lo),
                                                           o[i], 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[x][i]), p[x], o[i],
                                                            0, 0, 0);
    }
    settle(o[D / 16 - 1]);          // the last one issued
}

template <int kDtype>
__device__ inline float value_at(const uint32_t* w, int i) {
    if constexpr (kDtype == STAR_F32) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
}

// a / b of two counts: 64-bit divisions, a hundred instructions and more each,
// only where the counts need them
__device__ inline int64_t quotient(int64_t a, int64_t b) {
    if ((a | b) >> 32) return a / b;
    return (uint32_t)a / (uint32_t)b;
}

// ---------------------------------------------------------------------------
// The row-block kernel: any lengths, group sizes, masks and both types.
//
// A block is up to 16 (new token, query head) rows of one request that share a
// key-value head; its keys go by in tiles, one tile per wave and step, with
// the running maximum and sum of the softmax.  All blocks' steps in a row are
// cut into equal pieces, one per workgroup, whatever the requests' lengths: a
// piece ends inside a long cache or spans several short ones.  A block cut
// between workgroups leaves its parts (maximum, sum, unnormalised output) in
// the workspace, and the last of them to arrive joins all in order, so results
// do not depend on the order of arrival.  Keys and values are read once (16
// rows or fewer a head), registers to registers; HBM bounds it.
// ---------------------------------------------------------------------------
template <int kDtype, int D, bool kOnce>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attend_rows_kernel(AttendArgs a) {
    using TT = Tile<kDtype, D>;
    constexpr int kB = TT::kB, kT = TT::kT, E = TT::E;
    constexpr bool kAhead = D * kB < 1024;
    constexpr int kPart = kRows * D + 4 * kRows;       // floats of one part
    __shared__ float s_o[kWaves][kRows][D + 4];
    __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
    __shared__ int64_t s_tmp[2 * kWaves], s_steps[kThreads + 1], s_short[kThreads + 1];
    __shared__ Slot s_slot[kThreads];
    __shared__ uint32_t s_ticket;

    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int r = lane & 15, c = lane >> 4;
    const int wg = blockIdx.x;

    // steps of all blocks, and how many blocks have one step (`per` requests a
    // thread)
    const int per = (a.n_seq + kThreads - 1) / kThreads;
    int32_t bad = 0;
    {
        int64_t steps = 0, one = 0;
        for (int b = tid * per; b < min(a.n_seq, (tid + 1) * per); ++b) {
            const Slot s = slot_of<kT>(a, b, bad);
            if (per == 1) s_slot[tid] = s;
            const int64_t blocks = (int64_t)a.n_kv * s.blocks;
            steps += blocks * s.steps;
            one += s.steps == 1 ? blocks : 0;
        }
        if (wg == 0) report_error(a.err, bad);
        int64_t x = steps, y = one;
        block_incl_add2_i64<kThreads>(x, y, s_tmp);
        s_steps[tid] = x - steps, s_short[tid] = y - one;
        if (tid == kThreads - 1) s_steps[kThreads] = x, s_short[kThreads] = y;
        __syncthreads();
    }
    // Where they fill the chip by themselves, blocks of one step are a wave's
    // each (in batches of short requests three waves of four had no tile, and
    // every block cost a meeting: 512 requests of 30 tokens took 52 us, now 23)
    const int64_t n_short = s_short[kThreads] >= 2 * gridDim.x ? s_short[kThreads] : 0;
    const bool alone_too = n_short > 0;
    // the request that holds step (or one-step block) `at`, and its first
    struct Place {
        Slot s;
        int b;
        int64_t base, n;
    };
    auto find = [&](int64_t at, bool one) {
        auto before = [&](int i) {
            return one ? s_short[i] : s_steps[i] - (alone_too ? s_short[i] : 0);
        };
        auto width = [&](const Slot& s) {
            const int64_t blocks = (int64_t)a.n_kv * s.blocks;
            return one ? (s.steps == 1 ? blocks : 0)
                       : alone_too && s.steps == 1 ? 0 : blocks * s.steps;
        };
        int chunk = -1;                  // the last that starts at or before `at`
        for (int q = 0; q < min(a.n_seq, kThreads); q += kWave)
            chunk += __popcll(__ballot(q + lane < a.n_seq && before(q + lane) <= at));
        chunk = __builtin_amdgcn_readfirstlane(chunk);
        Place x;
        x.base = readlane_i64(before(chunk), 0);
        if (per == 1) {
            x.b = chunk;
            x.s.L = __builtin_amdgcn_readfirstlane(s_slot[chunk].L);
            x.s.T = __builtin_amdgcn_readfirstlane(s_slot[chunk].T);
            x.s.row0 = __builtin_amdgcn_readfirstlane(s_slot[chunk].row0);
            x.s.blocks = __builtin_amdgcn_readfirstlane(s_slot[chunk].blocks);
            x.s.steps = __builtin_amdgcn_readfirstlane(s_slot[chunk].steps);
            x.n = width(x.s);
            return x;
        }
        x.n = 0;
        x.b = 0;
        x.s = Slot{0, 0, 0, 0, 0};
        const int end = min(a.n_seq, (chunk + 1) * per);
        for (int from = chunk * per; from < end; from += kWave) {
            Slot s = {0, 0, 0, 0, 0};
            int32_t ignored = 0;
            if (from + lane < end) s = slot_of<kT>(a, from + lane, ignored);
            const int64_t mine = width(s);
            const int64_t upto = wave_incl_add_i64(mine);
            const uint64_t past = __ballot(x.base + upto > at);
            if (past) {
                const int i = __builtin_ctzll(past);
                x.b = from + i;
                x.base += readlane_i64(upto - mine, i);
                x.n = readlane_i64(mine, i);
                x.s.L = __builtin_amdgcn_readlane(s.L, i);
                x.s.T = __builtin_amdgcn_readlane(s.T, i);
                x.s.row0 = __builtin_amdgcn_readlane(s.row0, i);
                x.s.blocks = __builtin_amdgcn_readlane(s.blocks, i);
                x.s.steps = __builtin_amdgcn_readlane(s.steps, i);
                break;
            }
            x.base += readlane_i64(upto, kWave - 1);
        }
        return x;
    };

    // this workgroup's piece of the other blocks' steps
    const int64_t total = s_steps[kThreads] - n_short;
    const int64_t piece = max((int64_t)1, quotient(total + gridDim.x - 1, gridDim.x));
    int64_t u = wg * piece;
    const int64_t end = min(total, u + piece);
    int64_t k = wg + (int64_t)wave * gridDim.x;          // this wave's next one-step block
    int32_t err = 0;
    Place at_slot;
    at_slot.base = at_slot.n = 0;

    const __amdgpu_buffer_rsrc_t part =
        xch_rsrc(a.part, (uint32_t)(2 * gridDim.x * kPart * sizeof(float)));
    for (;;) {
        const bool together = u < end;                   // all four waves, else one
        if (!together && k >= n_short) break;
        if (!together || u >= at_slot.base + at_slot.n)
            at_slot = find(together ? u : k, !together);
        const Slot s = at_slot.s;
        const int b = at_slot.b;
        const int64_t base = at_slot.base;
        const int item = together ? (int)quotient(u - base, s.steps) : (int)(k - base);
        const int64_t item_u = base + (int64_t)item * s.steps;
        const int step0 = together ? (int)(u - item_u) : 0;
        const int steps = together ? (int)min((int64_t)(s.steps - step0), end - u) : 1;
        const int head = item / s.blocks, row_from = (item - head * s.blocks) * kRows;
        const int rows = min(s.T * a.g - row_from, kRows);

        // lane (r, c)'s row: its query and the position it stands at
        const int first = s.L - s.T;                     // position of the first new token
        const int row = row_from + r;
        const bool live = r < rows && s.L > 0;
        const int pos = live ? first + row / a.g : -1;
        const int p0 = first + row_from / a.g;
        const int p1 = first + (row_from + rows - 1) / a.g;
        const int64_t q_row = s.row0 + row / a.g;
        const int q_head = head * a.g + row % a.g;
        u32x4 q[TT::kChunks];
        if (live) {
            load_k<kDtype, D>(a.q + q_row * a.q_stride + (int64_t)q_head * D * kB, c, q);
        } else {
#pragma unroll
            for (int i = 0; i < TT::kChunks; ++i) q[i] = u32x4{0, 0, 0, 0};
        }

        const Tiles tl = tiles_of<kT>(a, p0, s.L > 0 ? p1 : -1);
        const int32_t* pages = a.table + (int64_t)b * a.max_pages;
        // the new tokens come from their own arrays (row 0: position `first`):
        // the cache is written beside, and no one reads them there
        const char* kn = a.kn + (int64_t)s.row0 * a.kv_stride + (int64_t)head * D * kB;
        const char* vn = a.vn + (int64_t)s.row0 * a.kv_stride + (int64_t)head * D * kB;
        const int64_t v_off = (int64_t)a.n_kv * D * kB << a.ps_log2;   // values after keys

        // where half h of tile t lies; a half that no row of the block sees is
        // not looked up (its page may be gone), and a bad page is left out
        auto half_at = [&](int t, int h) {
            Half x;
            const int j = t * kT + h * 16;
            const bool seen = j <= p1 && (!a.window || j + 15 > p0 - a.window || j < a.sinks);
            int page = 0;
            if (seen) page = pages[j >> a.ps_log2];
            page = __builtin_amdgcn_readfirstlane(page);
            x.ok = seen && (uint32_t)page < (uint32_t)a.n_pages;
            if (seen && !x.ok) err |= STAR_DEV_BAD_PAGE;
            const int in = j & ((1 << a.ps_log2) - 1);
            x.base = a.kv + (int64_t)(x.ok ? page : 0) * a.page_stride +
                     (((int64_t)head << a.ps_log2) + in) * (D * kB);
            return x;
        };
        auto load = [&](int t, TT& f, Half (&hf)[TT::kHalves]) {
#pragma unroll
            for (int h = 0; h < TT::kHalves; ++h) {
                hf[h] = half_at(t, h);
                const char* kb = hf[h].base + r * (D * kB);
                const char* vb = hf[h].base + v_off + c * 4 * (D * kB) + r * TT::kRowV;
                const int j = t * kT + h * 16;
                if (j + 16 > first && s.L > 0) {
                    auto row_at = [&](const char* rows, int token, const char* cached) {
                        return token < first ? cached
                                             : rows + (int64_t)(min(token, s.L - 1) - first) *
                                                          a.kv_stride;
                    };
                    load_k<kDtype, D>(row_at(kn, j + r, kb), c, f.k[h]);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        load_row<kDtype, D, kOnce>(row_at(vn + r * TT::kRowV, j + 4 * c + x,
                                                   vb + x * (D * kB)),
                                            f.v[4 * h + x]);
                } else {
                    load_k<kDtype, D>(kb, c, f.k[h]);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        load_row<kDtype, D, kOnce>(vb + x * (D * kB), f.v[4 * h + x]);
                }
            }
        };

        f32x4 o[E];
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        float m = -INFINITY, l = 0.0f;                   // l: this lane's tokens only

        const int t_step = together ? kWaves : 1;
        const int t_end = min(tl.n, kWaves * (step0 + steps));
        int t = together ? kWaves * step0 + wave : 0;
        TT f;
        Half hf[TT::kHalves];
        if (t < t_end) load(tl.at(t), f, hf);
        for (; t < t_end; t += t_step) {
            TT nf;
            Half nh[TT::kHalves];
            if (kAhead && t + t_step < t_end) load(tl.at(t + t_step), nf, nh);

            const int j0 = tl.at(t) * kT;
            float p[4 * TT::kHalves];
#pragma unroll
            for (int h = 0; h < TT::kHalves; ++h) {
                const f32x4 z = scores<kDtype, D>(f.k[h], q);
#pragma unroll
                for (int x = 0; x < 4; ++x) p[4 * h + x] = z[x] * a.scale_log2;
            }
            // hidden keys: only where the tile is not visible to every row
            bool all = j0 + kT - 1 <= p0 && rows == kRows;
            all = all && (!a.window || j0 > p1 - a.window || j0 + kT <= a.sinks);
#pragma unroll
            for (int h = 0; h < TT::kHalves; ++h) all = all && hf[h].ok;
            auto sees = [&](int j, int at, bool ok) {
                return ok && j <= at && (!a.window || j > at - a.window || j < a.sinks);
            };
            if (!all) {
#pragma unroll
                for (int h = 0; h < TT::kHalves; ++h)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int j = j0 + 16 * h + 4 * c + x;
                        if (!sees(j, pos, hf[h].ok)) p[4 * h + x] = -INFINITY;
                        // values that no row sees may be anything: 0 there
                        const bool any = hf[h].ok && j <= p1 &&
                                         (!a.window || j > p0 - a.window || j < a.sinks);
#pragma unroll
                        for (int w = 0; w < TT::kRowV / 4; ++w)
                            if (!any) f.v[4 * h + x][w] = 0;
                    }
            }
            // the tile's largest magnitude tells whether all values are finite
            uint32_t big = 0;
#pragma unroll
            for (int x = 0; x < TT::kRowsV; ++x)
#pragma unroll
                for (int w = 0; w < TT::kRowV / 4; ++w) big = larger<kDtype>(big, f.v[x][w]);

            float top = p[0];
#pragma unroll
            for (int x = 1; x < 4 * TT::kHalves; ++x) top = fmaxf(top, p[x]);
            top = fmaxf(m, quad_max(top));
            const float ref = top == -INFINITY ? 0.0f : top;   // nothing seen yet: all p are 0
            if (__any(top > m)) {
                const float f_old = __builtin_amdgcn_exp2f(m - ref);
                l *= f_old;
#pragma unroll
                for (int i = 0; i < E; ++i) o[i] *= f_old;
            }
            m = top;
#pragma unroll
            for (int x = 0; x < 4 * TT::kHalves; ++x) {
                p[x] = __builtin_amdgcn_exp2f(p[x] - ref);
                l += p[x];
            }
            // A value that is not finite would reach rows that do not see it as
            // 0 times infinity, and the rows that do as infinity times hi + lo
            // of unlike signs: such values leave the product and are added to
            // the rows that see them (their probabilities are positive)
            const bool fix = __any(not_finite<kDtype>(big));
            if (fix) {
                uint32_t* raw = (uint32_t*)&s_o[wave][0][0];     // [kT][D], as loaded
#pragma unroll
                for (int h = 0; h < TT::kHalves; ++h)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int w = 0; w < TT::kRowV / 4; ++w) {
                            uint32_t& v = f.v[4 * h + x][w];
                            raw[((16 * h + 4 * c + x) * D + r * E) * kB / 4 + w] = v;
                            v = finite_part<kDtype>(v);
                        }
            }
            accumulate<kDtype, D>(f.v, p, o);
            if (fix) {
                const uint32_t* raw = (const uint32_t*)&s_o[wave][0][0];
                for (int j = 0; j < kT; ++j) {
                    if (!sees(j0 + j, pos, j < 16 ? hf[0].ok : hf[TT::kHalves - 1].ok)) continue;
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            const float v = value_at<kDtype>(raw, j * D + (4 * c + x) * E + i);
                            if (!(fabsf(v) < INFINITY)) o[i][x] += v;
                        }
                }
            }

            if (kAhead) {
                f = nf;
#pragma unroll
                for (int h = 0; h < TT::kHalves; ++h) hf[h] = nh[h];
            } else if (t + t_step < t_end) {
                load(tl.at(t + t_step), f, hf);
            }
        }

        // new tokens join the cache with the block that holds their first row,
        // once per key-value head
        if (step0 == 0 && s.L > 0) {
            const int i0 = (row_from + a.g - 1) / a.g, i1 = (row_from + rows - 1) / a.g;
            constexpr int kPer = D * kB / 16;             // 16-byte pieces of a row
            for (int x = together ? tid : lane; x < (i1 - i0 + 1) * 2 * kPer;
                 x += together ? kThreads : kWave) {
                const int i = i0 + x / (2 * kPer), d = x % kPer * 16, j = first + i;
                const bool value = x / kPer & 1;
                const int page = pages[j >> a.ps_log2];
                if ((uint32_t)page < (uint32_t)a.n_pages)
                    *(u32x4*)(a.kv + (int64_t)page * a.page_stride + (value ? v_off : 0) +
                              (((int64_t)head << a.ps_log2) + (j & ((1 << a.ps_log2) - 1))) *
                                  (D * kB) +
                              d) =
                        *(const u32x4*)((value ? vn : kn) + (int64_t)i * a.kv_stride + d);
            }
        }

        l = quad_sum(l);
        if (!together) {
            // lane (r, c) has row r's outputs 4c E .. 4 (c + 1) E - 1
            if (r < rows) {
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // a row that sees nothing is 0
                const int64_t at = q_row * a.n_heads + q_head;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    float y[E];
#pragma unroll
                    for (int i = 0; i < E; ++i) y[i] = o[i][x] * inv;
                    store_out<kDtype, E>(a.out + (at * D + (4 * c + x) * E) * kB, y);
                }
                if (a.lse && c == 0)
                    a.lse[at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
            }
            k += (int64_t)kWaves * gridDim.x;
            continue;
        }

        // the four waves' parts meet: thread (row, 16 of them) sums E outputs
        if (c == 0) s_m[wave][r] = m, s_l[wave][r] = l;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int i = 0; i < E; ++i) s_o[wave][r][(4 * c + x) * E + i] = o[i][x];
        __syncthreads();
        const int jr = tid / 16, jd = (tid & 15) * E;
        float jm = s_m[0][jr], jl = 0.0f, jo[E];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) jm = fmaxf(jm, s_m[w][jr]);
        float jref = jm == -INFINITY ? 0.0f : jm;
#pragma unroll
        for (int i = 0; i < E; ++i) jo[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f_w = __builtin_amdgcn_exp2f(s_m[w][jr] - jref);
            jl += f_w * s_l[w][jr];
#pragma unroll
            for (int i = 0; i < E; ++i) jo[i] += f_w * s_o[w][jr][jd + i];
        }

        bool write = true;
        if (steps < s.steps) {
            // a part of a block: its place goes by the workgroup that holds it
            // (the block's first part after that workgroup's own first)
            const int w0 = (int)quotient(item_u, piece);
            const int w1 = (int)quotient(item_u + s.steps - 1, piece);
            auto part_at = [&](int w) {
                return (uint32_t)((2 * w + (w == w0)) * kPart * sizeof(float));
            };
            const uint32_t off = part_at(wg);
            if (jr < rows) {
                if ((tid & 15) == 0)
                    xch_store(u32x4{__float_as_uint(jm), __float_as_uint(jl), 0, 0}, part,
                              off + jr * 16);
#pragma unroll
                for (int i = 0; i < E; i += 4)
                    xch_store(u32x4{__float_as_uint(jo[i]), __float_as_uint(jo[i + 1]),
                                    __float_as_uint(jo[i + 2]), __float_as_uint(jo[i + 3])},
                              part, off + kRows * 16 + (jr * D + jd + i) * 4);
            }
            xch_wait_stores();
            write = xch_last_arrival(a.tickets + w0, (uint32_t)(w1 - w0 + 1), &s_ticket);
            if (write) {
                // In order, several parts' loads in flight, and where the block
                // has few rows, the threads of the others take every second (4th,
                // ..) part: one at a time cost 0.5 us each, 30 us for a long cache
                // cut 64 times
                constexpr int kBatch = D == 64 ? 4 : 2;
                const int lg = rows > 8 ? 4 : rows > 4 ? 3 : rows > 2 ? 2 : rows > 1 ? 1 : 0;
                const int groups = kRows >> lg, group = jr >> lg, pr = jr & ((1 << lg) - 1);
                jm = -INFINITY, jl = 0.0f;
#pragma unroll
                for (int i = 0; i < E; ++i) jo[i] = 0.0f;
                for (int w = w0 + group; w <= w1; w += kBatch * groups) {
                    u32x4 ml[kBatch], v[kBatch][E / 4];
#pragma unroll
                    for (int x = 0; x < kBatch; ++x) {
                        const int wx = w + x * groups;
                        const uint32_t at = wx <= w1 ? part_at(wx) : kXchOob;
                        ml[x] = xch_load(part, at + pr * 16);
#pragma unroll
                        for (int i = 0; i < E; i += 4)
                            v[x][i / 4] = xch_load(part, at + kRows * 16 + (pr * D + jd + i) * 4);
                    }
                    float top = jm;
#pragma unroll
                    for (int x = 0; x < kBatch; ++x)
                        if (w + x * groups <= w1) top = fmaxf(top, __uint_as_float(ml[x][0]));
                    jref = top == -INFINITY ? 0.0f : top;
                    const float f0 = __builtin_amdgcn_exp2f(jm - jref);
                    jm = top;
                    jl *= f0;
#pragma unroll
                    for (int i = 0; i < E; ++i) jo[i] *= f0;
#pragma unroll
                    for (int x = 0; x < kBatch; ++x) {
                        if (w + x * groups > w1) break;
                        const float f1 = __builtin_amdgcn_exp2f(__uint_as_float(ml[x][0]) - jref);
                        jl += __uint_as_float(ml[x][1]) * f1;
#pragma unroll
                        for (int i = 0; i < E; ++i)
                            jo[i] += __uint_as_float(v[x][i / 4][i & 3]) * f1;
                    }
                }
                if (groups > 1) {
                    // (every thread has read the waves' parts: the meeting is past)
                    if ((tid & 15) == 0) s_m[0][jr] = jm, s_l[0][jr] = jl;
#pragma unroll
                    for (int i = 0; i < E; ++i) s_o[0][jr][jd + i] = jo[i];
                    __syncthreads();
                    if (jr < rows) {
                        for (int x = 1; x < groups; ++x) jm = fmaxf(jm, s_m[0][(x << lg) + jr]);
                        jref = jm == -INFINITY ? 0.0f : jm;
                        jl = 0.0f;
#pragma unroll
                        for (int i = 0; i < E; ++i) jo[i] = 0.0f;
                        for (int x = 0; x < groups; ++x) {
                            const float f1 =
                                __builtin_amdgcn_exp2f(s_m[0][(x << lg) + jr] - jref);
                            jl += f1 * s_l[0][(x << lg) + jr];
#pragma unroll
                            for (int i = 0; i < E; ++i)
                                jo[i] += f1 * s_o[0][(x << lg) + jr][jd + i];
                        }
                    }
                }
            }
        }
        if (write && jr < rows) {
            const int wr = row_from + jr;
            const int64_t at = (int64_t)(s.row0 + wr / a.g) * a.n_heads + head * a.g + wr % a.g;
            const float inv = jl == 0.0f ? 0.0f : 1.0f / jl;   // a row that sees nothing is 0
#pragma unroll
            for (int i = 0; i < E; ++i) jo[i] *= inv;
            store_out<kDtype, E>(a.out + (at * D + jd) * kB, jo);
            if (a.lse && (tid & 15) == 0)
                a.lse[at] = jl == 0.0f ? -INFINITY : (jm + __builtin_amdgcn_logf(jl)) * kLn2;
        }
        __syncthreads();                                  // s_o is free for the next block
        u += steps;
    }
    if (err && lane == 0) report_error(a.err, err);
}

template <int kDtype, int D>
hipError_t launch_rows(const AttendArgs& a, int grid, hipStream_t stream) {
    // one block a request and key-value head reads every key and value once
    if (!a.q_start && a.g <= kRows)
        hipLaunchKernelGGL((attend_rows_kernel<kDtype, D, true>), dim3(grid), dim3(kThreads), 0,
                           stream, a);
    else
        hipLaunchKernelGGL((attend_rows_kernel<kDtype, D, false>), dim3(grid), dim3(kThreads), 0,
                           stream, a);
    return hipGetLastError();
}

}  // namespace

AttendPlan plan_attend(const star_attend_params& p, bool decode) {
    AttendPlan pl;
    // two workgroups a CU (one where a row's 256 elements fill the registers; 64 wide
    // a third would fit)
    pl.grid = p.head_dim == 256 ? 256 : 512;
    static_assert(512 <= kMaxTickets, "one ticket per workgroup");
    pl.part_bytes = (size_t)2 * pl.grid * (kRows * p.head_dim + 4 * kRows) * sizeof(float);
    if (!decode) plan_attend_tiles(p, pl);
    return pl;
}

hipError_t launch_attend(const AttendPlan& pl, const AttendArgs& args, int dtype, int head_dim,
                         hipStream_t stream) {
    AttendArgs a = args;
    a.splits = pl.splits;
    a.part_tiles = pl.part_tiles;
    a.items = pl.items;
    if (a.n_seq == 0 || a.n_rows == 0) return hipSuccess;
    if (pl.tiled) return launch_attend_tiles(a, dtype, head_dim, stream);
    if (dtype == STAR_BF16) {
        if (head_dim == 64) return launch_rows<STAR_BF16, 64>(a, pl.grid, stream);
        if (head_dim == 128) return launch_rows<STAR_BF16, 128>(a, pl.grid, stream);
        return launch_rows<STAR_BF16, 256>(a, pl.grid, stream);
    }
    if (head_dim == 64) return launch_rows<STAR_F32, 64>(a, pl.grid, stream);
    if (head_dim == 128) return launch_rows<STAR_F32, 128>(a, pl.grid, stream);
    return launch_rows<STAR_F32, 256>(a, pl.grid, stream);
}

}  // namespace star
