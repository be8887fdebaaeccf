// Attention of many new tokens over the paged key-value cache: the kernel of
// star_attend_prompt whose keys and values go through LDS.
#include <algorithm>

#include "attend.hpp"
#include "star_common.hpp"
#include "star_internal.hpp"

namespace star {

namespace {

constexpr int kBM = 128;         // query rows of a workgroup, 32 a wave
constexpr int kThreads = 256, kWaves = 4;
// workgroups that run at once, two a CU: the 128-wide and fp32 kernels' (64 wide in
// bf16 three fit, 256 wide one)
constexpr int kPlaces = 512;
constexpr int kMaxParts = 8;     // parts of a block's keys at most
constexpr int kMoreParts = 512;  // of a launch's longer blocks, beside those the host counts
constexpr int kPartTiles = 16;   // and the fewest tiles of one: shorter ones do not pay
constexpr float kLazy = 8.0f;    // log2 of the factor that a stale maximum may lag

typedef __attribute__((address_space(3))) char* lds_t;
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int kDtype, int D>
struct Lay {
    static constexpr int kBytes = kDtype == STAR_BF16 ? 2 : 4;
    static constexpr int kRow = kBytes * D;       // bytes of a token's keys (or values)
    // tokens of a tile, a quarter a wave to load (two workgroups' tiles fit LDS;
    // where a row fills the registers, one workgroup's do)
    static constexpr int kBN = kRow > 256 ? 32 : 64;
    static constexpr int kPages = kBN / 16;       // sixteens of tokens, each in one page
    static constexpr int kLoadRows = kBN / 4;     // tokens that a wave loads
    static constexpr int kChunks = kRow / 16;     // 16-byte chunks of a row
    static constexpr int kTile = kBN * kRow;      // bytes of a tile's keys
    static constexpr int kRowsPerLoad = 1024 / kRow;
    static constexpr int kLoads = kLoadRows / kRowsPerLoad;   // 1 KiB loads of those
    // Chunk c of row r lies at chunk c ^ f(r) of the row.  Keys: 16 lanes read
    // one chunk of 16 rows; bf16 values: 32 lanes read 32 bytes of 4 rows and the
    // 32 bytes beside; fp32 values: 32 lanes 128 bytes of a row, the others of the
    // fourth row on; in each case every bank is read once.
    __device__ static int fk(int r) { return kRow == 128 ? (r >> 1) & 7 : r & 15; }
    __device__ static int fv(int r) {
        if (kDtype == STAR_F32) return ((r >> 2) & 1) * 8;
        return kRow == 128 ? ((r >> 1) & 1) * 4 : (r & 3) * 4;
    }
};

// the maximum of lanes l and l ^ 32
__device__ inline float pair_max(float v) {
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ inline float pair_sum(float v) {
    auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// floats a thread leaves in a part: its outputs, maximum and sum (padded)
template <int D>
constexpr int kPartFloats = D / 2 + 4;

// ---------------------------------------------------------------------------
// One workgroup: 128 (token, query head) rows of one request that share a
// key-value head, tokens before heads, so that a group's heads share every
// tile.  Lane l of a wave owns row l % 32: S^T [tokens x rows] = K Q^T gives it
// the scores of half the tokens, its exponentials are in place as the second
// operand of O^T [d x rows] = V^T P^T, and the softmax needs one exchange with
// lane l ^ 32 a tile.  V's fragments are read from LDS transposed.
// ---------------------------------------------------------------------------
template <int kDtype, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attend_tiles_kernel(AttendArgs a) {
    using Y = Lay<kDtype, D>;
    constexpr bool kBf16 = kDtype == STAR_BF16;
    constexpr int kSteps = Y::kRow / 32; // 32-byte steps of a score's contraction
    constexpr int kOut = D / 32;         // 32-wide blocks of the output
    constexpr int kBN = Y::kBN;
    __shared__ __attribute__((aligned(1024))) char s_kv[2][2][Y::kTile];
    __shared__ int64_t s_tmp[kWaves + 1];
    __shared__ int s_slot[2], s_fix[2];
    __shared__ uint32_t s_ticket;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int r32 = lane & 31, half = lane >> 5;

    // which request, which of its blocks of rows and which part of the block's keys:
    // those with the longest prefixes first, so that the launch ends on short ones
    const int head = blockIdx.x % a.n_kv, item = blockIdx.x / a.n_kv;
    int b, block, nth, part = 0, parts = 1;
    if (a.n_seq <= 64) {
        // One request a lane, every wave by itself.  More requests run in reverse order,
        // with one number of parts: that takes 64 unlike chunks after up to 3000 tokens
        // from 164 to 189 us, 60 of 40 tokens after up to 8000 from 161 to 207, one prompt
        // of 2000 among 63 of 20 from 83 to 91, and 64 equal prompts of 300 from 226 to 212
        int32_t bad = 0;
        Slot s = {0, 0, 0, 0, 0};
        if (lane < a.n_seq) s = slot_of<kBN>(a, lane, bad);
        if (blockIdx.x == 0 && wave == 0) report_error(a.err, bad);
        const int n = (s.T * a.g + kBM - 1) / kBM;
        // the request's blocks whose last position is X or more
        auto reach = [&](int x) {
            const int t = x - (s.L - s.T);
            return t <= 0 ? n : t >= s.T ? 0 : n - (t * a.g >> 7);
        };
        static_assert(kBM == 128, "reach divides by it");
        auto all = [&](int mine) {
            return __builtin_amdgcn_readlane(wave_incl_add_i32(mine), 63);
        };
        // Where the host cuts at all: blocks with a last position of X or more have
        // k parts or more, for an X that grows with k; count[k] of them, the first in
        // the order, so that no workgroup is without work (4 requests of 600 after 0 to
        // 6000 tokens: 247 us where a block's spare parts ended early, now 200).  A
        // block is cut as the host says, or into more where it is longer than a place's
        // fair share of all tiles (3 requests of 300 after 0 to 16000: 217 -> 182); the
        // share grows until the parts fit the launch.
        int count[kMaxParts + 2] = {};
        count[1] = all(n);
        int64_t sum = count[1];
        const int cap = a.window && a.sinks < (1 << 30) - a.window ? a.window + a.sinks : 1 << 30;
        auto tiles = [&](int x) { return min(x, cap) / kBN; };
        if (a.splits > 1 && __any(tiles(s.L) >= 2 * kPartTiles)) {
            int64_t total = (int64_t)n * ((tiles(s.L - s.T) + tiles(s.L)) / 2 + 1);
            total = readlane_i64(wave_incl_add_i64(total), 63) * a.n_kv /
                    (D == 256 ? kPlaces / 2 : kPlaces);
            constexpr int kMost = 1 << 26;
            int share = (int)min((int64_t)kMost, max((int64_t)kPartTiles, total));
            for (;; share *= 2) {
                sum = count[1];
#pragma unroll
                for (int k = 2; k <= kMaxParts; ++k) {
                    int least = max(kPartTiles * k, (k - 1) * share + 1);
                    if (k <= a.splits) least = min(least, a.part_tiles * k);
                    count[k] = least > cap / kBN ? 0 : all(reach(least * kBN - 1));
                    sum += count[k];
                }
                if (sum <= a.items && (int64_t)count[2] * a.n_kv <= kMaxTickets) break;
                if (share >= kMost) {          // (only where ranges of rows overlap)
#pragma unroll
                    for (int k = 2; k <= kMaxParts; ++k) count[k] = 0;
                    sum = count[1];
                    break;
                }
            }
        }
        if (item >= sum) return;
        nth = item;
        int at = item;
#pragma unroll
        for (int k = kMaxParts; k > 0; --k) {
            const int here = (count[k] - count[k + 1]) * k;      // parts of blocks of k
            if (at >= 0 && at < here) nth = count[k + 1] + at / k, part = at % k, parts = k;
            at -= here;
        }
        // the largest last position X that more than nth blocks reach, then the
        // blocks at X in order
        int lo = 0, hi = 64;
        while (__any(hi < s.L)) hi <<= 1;                // (L is at most 2^30)
        while (hi - lo > 1) {
            const int mid = lo + (hi - lo) / 2;
            if (all(reach(mid)) > nth) lo = mid;
            else hi = mid;
        }
        const int rank = nth - all(reach(lo + 1)), here = reach(lo) - reach(lo + 1);
        const int upto = wave_incl_add_i32(here);
        const uint64_t past = __ballot(upto > rank);
        b = __builtin_ctzll(past);
        block = __builtin_amdgcn_readlane(n - reach(lo) + rank - (upto - here), b);
    } else {
        nth = item / a.splits, part = item - nth * a.splits;
        const int per = (a.n_seq + kThreads - 1) / kThreads;
        int64_t mine = 0, total;
        int32_t bad = 0;
        auto blocks = [&](int x) { return (slot_of<kBN>(a, x, bad).T * a.g + kBM - 1) / kBM; };
        for (int x = tid * per; x < min(a.n_seq, (tid + 1) * per); ++x) mine += blocks(x);
        if (blockIdx.x == 0) report_error(a.err, bad);
        const int64_t before =
            block_exclusive_scan_i64<kThreads>(mine, OpAdd(), 0, s_tmp, &total);
        const int64_t at = total - 1 - nth;
        if (at < 0) return;
        if (before <= at && at < before + mine) {
            int64_t base = before;
            for (int x = tid * per;; ++x) {
                const int n = blocks(x);
                if (at < base + n) {
                    s_slot[0] = x;
                    s_slot[1] = (int)(at - base);
                    break;
                }
                base += n;
            }
        }
        __syncthreads();
        b = __builtin_amdgcn_readfirstlane(s_slot[0]);
        block = __builtin_amdgcn_readfirstlane(s_slot[1]);
    }
    int32_t ignored = 0;
    const Slot s = slot_of<kBN>(a, b, ignored);
    const int all_rows = s.T * a.g;                  // (below 2^31 over all requests)
    const int row_from = block * kBM;
    const int first = s.L - s.T;
    auto pos_of = [&](int row) { return first + min(row, all_rows - 1) / a.g; };
    const int p0 = pos_of(row_from), p1 = pos_of(row_from + kBM - 1);       // the workgroup's
    const int wave_row = row_from + 32 * wave;
    const int w0 = pos_of(wave_row), w1 = pos_of(wave_row + 31);            // the wave's
    const bool live = wave_row + r32 < all_rows;
    const int row = min(wave_row + r32, all_rows - 1);
    const int pos = live ? first + row / a.g : -1;
    const int64_t q_row = s.row0 + row / a.g;
    const int q_head = head * a.g + row % a.g;

    // a negative scale turns the queries' signs, so that the largest score is
    // the largest product; a scale of 0 is the least number, so that hidden keys'
    // -infinity stays what it is
    const float c = fmaxf(fabsf(a.scale_log2), 0x1p-126f);
    const uint32_t turn = a.scale_log2 < 0.0f ? (kBf16 ? 0x80008000u : 0x80000000u) : 0u;
    u32x4 q[kSteps];
    {
        const char* p = a.q + q_row * a.q_stride + (int64_t)q_head * Y::kRow + half * 16;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            q[i] = live ? *(const u32x4*)(p + 32 * i) : u32x4{0, 0, 0, 0};
            q[i] ^= turn;
        }
    }

    const int32_t* pages = a.table + (int64_t)b * a.max_pages;
    const Tiles tl = tiles_of<kBN>(a, p0, p1);
    // this workgroup's share of the tiles: all, or one of `parts`
    if (a.n_seq > 64) parts = max(1, min(a.splits, tl.n / a.part_tiles));
    if (part >= parts) return;
    const int u0 = (int)((int64_t)tl.n * part / parts);
    const int u1 = (int)((int64_t)tl.n * (part + 1) / parts);
    const int64_t v_off = (int64_t)a.n_kv * Y::kRow << a.ps_log2;
    const int64_t head_off = (int64_t)head * Y::kRow << a.ps_log2;
    int32_t err = 0;

    // lane x % kPages' sixteen tokens of a tile: their page, or -1 where no row of
    // the workgroup sees one of them; a bad page reports and reads page 0
    struct Pages {
        int page;
        bool ok;
    };
    auto look_up = [&](int u) {
        const int j = tl.at(u) * kBN + 16 * (lane & (Y::kPages - 1));
        const bool seen = j <= p1 && (!a.window || j + 15 > p0 - a.window || j < a.sinks);
        return seen ? pages[j >> a.ps_log2] : -1;
    };
    auto check = [&](int u, int page) {
        const int j = tl.at(u) * kBN + 16 * (lane & (Y::kPages - 1));
        const bool seen = j <= p1 && (!a.window || j + 15 > p0 - a.window || j < a.sinks);
        Pages x;
        x.ok = seen && (uint32_t)page < (uint32_t)a.n_pages;
        if (seen && !x.ok) err |= STAR_DEV_BAD_PAGE;
        x.page = x.ok ? page : 0;
        return x;
    };
    // this wave's tokens of a tile: keys and values into registers,
    // and from there into a buffer once the one before it is done with
    const int st_row = lane / Y::kChunks, st_ch = lane % Y::kChunks;
    const int g_off = st_row * Y::kRow + st_ch * 16;
    u32x4 next_k[Y::kLoads], next_v[Y::kLoads];
    auto address = [&](int u, const Pages& x) {
        const int page = __builtin_amdgcn_readlane(x.page, wave * Y::kLoadRows / 16);
        const int in = (tl.at(u) * kBN + Y::kLoadRows * wave) & ((1 << a.ps_log2) - 1);
        return a.kv + (int64_t)page * a.page_stride + head_off + (int64_t)in * Y::kRow + g_off;
    };
    auto load = [&](const char* base, u32x4 (&to)[Y::kLoads]) {
#pragma unroll
        for (int i = 0; i < Y::kLoads; ++i) to[i] = *(const u32x4*)(base + 1024 * i);
    };
    auto store_k = [&](int to) {
#pragma unroll
        for (int i = 0; i < Y::kLoads; ++i) {
            const int rr = i * Y::kRowsPerLoad + st_row;
            const int in_tile = wave * Y::kLoadRows + rr;
            *(u32x4*)(&s_kv[to][0][0] + in_tile * Y::kRow + (st_ch ^ Y::fk(in_tile)) * 16) =
                next_k[i];
        }
    };
    // values of a tile that not every row sees: those that are not finite
    // would reach the other rows as 0 times infinity, so they stay out of LDS,
    // and the tile is marked (by its number, so that no mark needs clearing)
    auto store_v = [&](int to, int u, bool plain) {
        if (!plain) {
            uint32_t big = 0;
#pragma unroll
            for (int i = 0; i < Y::kLoads; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) big = larger<kDtype>(big, next_v[i][x]);
            if (__any(not_finite<kDtype>(big))) {
#pragma unroll
                for (int i = 0; i < Y::kLoads; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        next_v[i][x] = finite_part<kDtype>(next_v[i][x]);
                s_fix[to] = u;
            }
        }
#pragma unroll
        for (int i = 0; i < Y::kLoads; ++i) {
            const int rr = i * Y::kRowsPerLoad + st_row;
            const int in_tile = wave * Y::kLoadRows + rr;
            *(u32x4*)(&s_kv[to][1][0] + in_tile * Y::kRow + (st_ch ^ Y::fv(in_tile)) * 16) =
                next_v[i];
        }
    };

    f32x16 o[kOut];
#pragma unroll
    for (int i = 0; i < kOut; ++i)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[i][x] = 0.0f;
    float m = -INFINITY, l = 0.0f;      // l: this lane's tokens only

    // lane addresses of the fragments in a tile
    const int k_base = r32 * Y::kRow, k_x = (half ^ Y::fk(r32)) * 16;
    const int i16 = lane & 15;
    const int v_base = kBf16 ? (4 * half + (i16 >> 2)) * Y::kRow + ((lane >> 4) & 1) * 32 +
                                   (i16 & 3) * 8
                             : 4 * half * Y::kRow + r32 * 4;
    // (fv depends on a row's bits below 8 alone, and the fragments' first rows are
    // multiples of 8; a 32-wide block of the output is a whole number of its steps)
    const int v_x = (kBf16 ? Y::fv(i16 >> 2) : 8 * half) * 16;

    // whether all tokens of a tile are visible to all rows from p to p_last
    auto plain_to = [&](int u, uint32_t ok4, int p, int p_last) {
        const int j0 = tl.at(u) * kBN;
        return ok4 == (1u << Y::kPages) - 1 && j0 + kBN - 1 <= p &&
               (!a.window || j0 > p_last - a.window || j0 + kBN <= a.sinks);
    };

    Pages now = check(u0, look_up(u0));
    uint32_t ok4 = (uint32_t)__ballot(now.ok) & ((1u << Y::kPages) - 1);
    if (tid < 2) s_fix[tid] = -1;
    __syncthreads();
    {
        const char* from = address(u0, now);
        load(from, next_k);
        load(from + v_off, next_v);
        store_k(u0 & 1);
        store_v(u0 & 1, u0, plain_to(u0, ok4, p0, p1));
    }
    int page_next = look_up(min(u0 + 1, u1 - 1));
    // the second wave of a SIMD goes first where both could: the two drift into
    // opposite phases, one's products beside the other's softmax
    if (__builtin_amdgcn_s_getreg(3 << 11 | 4) & 1) __builtin_amdgcn_s_setprio(1);
    for (int u = u0; u < u1; ++u) {
        __syncthreads();          // tile u is in its buffer, and the other one is done with
        const lds_t kb = (lds_t)&s_kv[u & 1][0][0], vb = (lds_t)&s_kv[u & 1][1][0];
        const int j0 = tl.at(u) * kBN;
        // (the last tile is loaded twice, so that no step hangs on a condition)
        const int un = min(u + 1, u1 - 1);
        const Pages here = now;
        const uint32_t ok_here = ok4;
        now = check(un, page_next);
        ok4 = (uint32_t)__ballot(now.ok) & ((1u << Y::kPages) - 1);
        const char* from = address(un, now);
        load(from, next_k);
        page_next = look_up(min(u + 2, u1 - 1));

        f32x16 z[kBN / 32];
#pragma unroll
        for (int t = 0; t < kBN / 32; ++t) {
#pragma unroll
            for (int x = 0; x < 16; ++x) z[t][x] = 0.0f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const u32x4 kf = *(__attribute__((address_space(3))) const u32x4*)(
                    kb + t * 32 * Y::kRow + k_base + ((32 * i) ^ k_x));
                if constexpr (kBf16) {
                    z[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        __builtin_bit_cast(bf16x8_t, kf), __builtin_bit_cast(bf16x8_t, q[i]), z[t],
                        0, 0, 0);
                } else {
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        z[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(
                            __uint_as_float(kf[x]), __uint_as_float(q[i][x]), z[t], 0, 0, 0);
                }
            }
        }
        load(from + v_off, next_v);
        auto sees = [&](int j) {
            return ((ok_here >> ((j - j0) >> 4)) & 1) && j <= pos &&
                   (!a.window || j > pos - a.window || j < a.sinks);
        };
#pragma unroll
        for (int t = 0; t < kBN / 32; ++t) settle(z[t]);
        if (!plain_to(u, ok_here, w0, w1)) {
#pragma unroll
            for (int t = 0; t < kBN / 32; ++t)
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    if (!sees(j0 + 32 * t + 8 * (x / 4) + 4 * half + x % 4)) z[t][x] = -INFINITY;
        }

        float top = z[0][0];
#pragma unroll
        for (int t = 0; t < kBN / 32; ++t)
#pragma unroll
            for (int x = 0; x < 16; ++x) top = fmaxf(top, z[t][x]);
        top = pair_max(top) * c;
        // the reference may lag the maximum by 2^kLazy: the sums have the room
        // (fp32), and bf16's relative step is the same everywhere
        if (__any(top > m + kLazy)) {
            const float peak = fmaxf(m, top);
            const float f = __builtin_amdgcn_exp2f(m - (peak == -INFINITY ? 0.0f : peak));
            m = peak;
            l *= f;
#pragma unroll
            for (int i = 0; i < kOut; ++i) o[i] *= f;
        }
        const float ref = m == -INFINITY ? 0.0f : m;      // nothing seen yet: all p are 0
        if constexpr (kBf16) {
            // One bf16 each, half a step (2^-8) off at most: the products share the time with
            // the softmax, and a hi + lo pair would double the second (8191 tokens
            // 610 -> 791 us, ragged prompts 323 -> 402; outputs then 1.65e-3 off instead
            // of 2.2e-3, 1.65e-3 of it their own rounding)
            u32x4 p[kBN / 16];            // 16 tokens each, as the second product takes them
#pragma unroll
            for (int t = 0; t < kBN / 32; ++t)
#pragma unroll
                for (int x = 0; x < 16; x += 2) {
                    const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][x], c, -ref));
                    const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][x + 1], c, -ref));
                    l += e0;
                    l += e1;
                    p[2 * t + x / 8][(x % 8) / 2] = pack_bf16x2_rne(e0, e1);
                }
            store_k((u + 1) & 1);
#pragma unroll
            for (int s4 = 0; s4 < kBN / 16; ++s4)
#pragma unroll
                for (int i = 0; i < kOut; ++i) {
                    const lds_t at = vb + v_base + s4 * 16 * Y::kRow + ((64 * i) ^ v_x);
                    typedef __attribute__((address_space(3))) s16x4* tr_t;
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)at);
                    const s16x4 hi =
                        __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(at + 8 * Y::kRow));
                    const u32x2 x0 = __builtin_bit_cast(u32x2, lo);
                    const u32x2 x1 = __builtin_bit_cast(u32x2, hi);
                    const u32x4 va = {x0[0], x0[1], x1[0], x1[1]};
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        __builtin_bit_cast(bf16x8_t, va), __builtin_bit_cast(bf16x8_t, p[s4]),
                        o[i], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int t = 0; t < kBN / 32; ++t)
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    z[t][x] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[t][x], c, -ref));
                    l += z[t][x];
                }
            store_k((u + 1) & 1);
            // element x of the two halves: tokens 8 (x / 4) + x % 4 and the fourth on
#pragma unroll
            for (int t = 0; t < kBN / 32; ++t)
#pragma unroll
                for (int x = 0; x < 16; ++x)
#pragma unroll
                    for (int i = 0; i < kOut; ++i)
                        o[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(
                            *(__attribute__((address_space(3))) const float*)(
                                vb + v_base + (32 * t + 8 * (x / 4) + x % 4) * Y::kRow +
                                ((128 * i) ^ v_x)),
                            z[t][x], o[i], 0, 0, 0);
        }
        if (s_fix[u & 1] == u) {
            // the values that were kept out reach the rows that see them (their
            // probabilities are positive), from the cache
#pragma unroll
            for (int i = 0; i < kOut; ++i) settle(o[i]);
            for (int j = 0; j < kBN; ++j) {
                const int page = __builtin_amdgcn_readlane(here.page, j >> 4);
                const char* raw = a.kv + (int64_t)page * a.page_stride + head_off + v_off +
                                  (int64_t)((j0 + j) & ((1 << a.ps_log2) - 1)) * Y::kRow +
                                  half * 4 * Y::kBytes;
                if (!sees(j0 + j)) continue;
#pragma unroll
                for (int i = 0; i < kOut; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const char* four = raw + (32 * i + 8 * x) * Y::kBytes;
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            float v;
                            if constexpr (kBf16)
                                v = __uint_as_float((uint32_t)((const uint16_t*)four)[y] << 16);
                            else
                                v = ((const float*)four)[y];
                            if (!(fabsf(v) < INFINITY)) o[i][4 * x + y] += v;
                        }
                    }
            }
        }
        store_v((u + 1) & 1, un == u ? -2 : un, plain_to(un, ok4, p0, p1));
    }
#pragma unroll
    for (int i = 0; i < kOut; ++i) settle(o[i]);
    if (err && lane < Y::kPages) report_error(a.err, err);

    l = pair_sum(l);
    if (parts > 1) {
        // The parts meet in the workspace, lane by lane as they are; the last to
        // arrive joins all in order
        constexpr uint32_t kPlane = kThreads * 16;               // 16 bytes a thread
        constexpr uint32_t kBytes = kPartFloats<D> * kThreads * 4;
        const uint32_t id = (uint32_t)(nth * a.n_kv + head);
        const __amdgpu_buffer_rsrc_t ws =
            xch_rsrc(a.part + ((size_t)head * a.items + (item - part)) * kBytes,
                     (uint32_t)parts * kBytes);
        const uint32_t mine = (uint32_t)part * kBytes + tid * 16;
        xch_store(u32x4{__float_as_uint(m), __float_as_uint(l), 0, 0}, ws, mine);
#pragma unroll
        for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int x = 0; x < 16; x += 4)
                xch_store(u32x4{__float_as_uint(o[i][x]), __float_as_uint(o[i][x + 1]),
                                __float_as_uint(o[i][x + 2]), __float_as_uint(o[i][x + 3])},
                          ws, mine + (1 + 4 * i + x / 4) * kPlane);
        xch_wait_stores();
        if (!xch_last_arrival(a.tickets + id, (uint32_t)parts, &s_ticket)) return;
        m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int i = 0; i < kOut; ++i)
#pragma unroll
            for (int x = 0; x < 16; ++x) o[i][x] = 0.0f;
        for (int w = 0; w < parts; ++w) {
            const uint32_t at = (uint32_t)w * kBytes + tid * 16;
            const u32x4 ml = xch_load(ws, at);
            u32x4 v[4 * kOut];
#pragma unroll
            for (int i = 0; i < 4 * kOut; ++i) v[i] = xch_load(ws, at + (1 + i) * kPlane);
            const float peak = fmaxf(m, __uint_as_float(ml[0]));
            const float ref = peak == -INFINITY ? 0.0f : peak;
            const float f0 = __builtin_amdgcn_exp2f(m - ref);
            const float f1 = __builtin_amdgcn_exp2f(__uint_as_float(ml[0]) - ref);
            m = peak;
            l = l * f0 + __uint_as_float(ml[1]) * f1;
#pragma unroll
            for (int i = 0; i < kOut; ++i)
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    o[i][x] = o[i][x] * f0 + __uint_as_float(v[4 * i + x / 4][x & 3]) * f1;
        }
    }
    if (!live) return;
    const int64_t at = q_row * a.n_heads + q_head;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;      // a row that sees nothing is 0
    char* to = a.out + at * Y::kRow + half * 4 * Y::kBytes;
#pragma unroll
    for (int i = 0; i < kOut; ++i)
#pragma unroll
        for (int x = 0; x < 16; x += 4) {
            const float y[4] = {o[i][x] * inv, o[i][x + 1] * inv, o[i][x + 2] * inv,
                                o[i][x + 3] * inv};
            store_out<kDtype, 4>(to + (32 * i + 2 * x) * Y::kBytes, y);
        }
    if (a.lse && half == 0)
        a.lse[at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---------------------------------------------------------------------------
// The new tokens of prompts into their pages, `rows` (at most 4) tokens a workgroup:
// a lane each finds their places, then all copy, 16 bytes a thread and several in
// flight.  Long calls take four (18 -> 13 us for 12700 tokens of 2 KB), whose
// places are looked up at once; short ones one, which starts sooner.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kThreads) void store_tokens_kernel(AttendArgs a, int row_bytes,
                                                                int rows) {
    __shared__ int64_t s_to[4];
    const int64_t row0 = (int64_t)blockIdx.x * rows;
    if ((int)threadIdx.x < rows) {
        const int64_t row = row0 + threadIdx.x;
        int64_t to = -1;
        // the request whose rows hold this one: the last that starts at or before it
        int lo = 0, hi = a.n_seq;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (a.q_start[mid] <= row) lo = mid + 1;
            else hi = mid;
        }
        const int b = lo - 1;
        if (b >= 0 && row < a.n_rows) {
            const int from = a.q_start[b], end = a.q_start[b + 1], L = a.seq_len[b];
            if (from >= 0 && row < end && end <= a.n_rows && L >= 0 &&
                L <= a.max_pages << a.ps_log2 && end - from <= L) {
                const int j = (int)(L - (end - from) + (row - from));
                const int page = a.table[(int64_t)b * a.max_pages + (j >> a.ps_log2)];
                if ((uint32_t)page < (uint32_t)a.n_pages)
                    to = (int64_t)page * a.page_stride +
                         (int64_t)(j & ((1 << a.ps_log2) - 1)) * row_bytes;
            }
        }
        s_to[threadIdx.x] = to;
    }
    __syncthreads();
    const int pieces = a.n_kv * row_bytes / 16;            // of one token's keys
    const int per = row_bytes / 16;                        // of one head's: 8, 16 or 32
    constexpr int kUnroll = 4;
    for (int x0 = threadIdx.x; x0 < rows * 2 * pieces; x0 += kUnroll * kThreads) {
        u32x4 v[kUnroll];
        char* to[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int x = x0 + u * kThreads, i = x / (2 * pieces), y = x - i * 2 * pieces;
            const bool value = y >= pieces;
            const int z = value ? y - pieces : y, head = z / per, d = (z - head * per) * 16;
            to[u] = nullptr;
            if (i < rows && s_to[i] >= 0) {
                v[u] = *(const u32x4*)((value ? a.vn : a.kn) + (row0 + i) * a.kv_stride +
                                       (int64_t)z * 16);
                to[u] = a.kv + s_to[i] +
                        ((int64_t)((value ? a.n_kv : 0) + head) << a.ps_log2) * row_bytes + d;
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (to[u]) *(u32x4*)to[u] = v[u];
    }
}

// an upper bound: every request has one block at most that is not full
int64_t tile_blocks(int64_t n_rows, int g, int n_seq) { return n_rows * g / kBM + n_seq; }

template <int kDtype, int D>
hipError_t launch_tiles(const AttendArgs& a, hipStream_t stream) {
    const int64_t grid = a.items * a.n_kv;
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    const int store = a.n_rows > 4096 ? 4 : 1;
    hipLaunchKernelGGL(store_tokens_kernel, dim3((a.n_rows + store - 1) / store), dim3(kThreads),
                       0, stream, a, Lay<kDtype, D>::kRow, store);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attend_tiles_kernel<kDtype, D>), dim3((unsigned)grid), dim3(kThreads), 0,
                       stream, a);
    return hipGetLastError();
}

template <int kDtype>
hipError_t launch_tiles_of(const AttendArgs& a, int head_dim, hipStream_t stream) {
    if (head_dim == 64) return launch_tiles<kDtype, 64>(a, stream);
    if constexpr (kDtype == STAR_BF16)
        if (head_dim == 256) return launch_tiles<kDtype, 256>(a, stream);
    return launch_tiles<kDtype, 128>(a, stream);
}

}  // namespace

void plan_attend_tiles(const star_attend_params& p, AttendPlan& pl) {
    const int g = p.n_heads / p.n_kv_heads;
    const int64_t rows = (int64_t)p.n_rows * g;
    const int e = p.dtype == STAR_BF16 ? 2 : 4;
    // workgroups, if the requests' last blocks are half full, and the most keys
    // that a row can see
    const int64_t groups = (rows + (int64_t)p.n_seq * kBM / 2) / kBM * p.n_kv_heads;
    int64_t keys = (int64_t)p.max_pages * p.page_size;
    if (p.window) keys = std::min(keys, (int64_t)p.window + p.sinks);
    // Only the host's numbers decide, so that a captured call keeps its kernel: the
    // table's width stands for the lengths, and n_rows / n_seq for a request's rows.
    // What that costs, both kernels measured: calls of single tokens, whose blocks hold
    // few rows, would be faster by row blocks (124 requests after up to 4000 tokens
    // 249 us against 211, 31 of them 71 against 56, with 16 heads of their own keys 127
    // against 158), as star_attend_decode takes them; but slots without rows and single
    // tokens beside a prompt look the same from here and lose more there (30 single
    // tokens and 2048 rows of one prompt 121 against 724, 256 and 512 rows 253 against
    // 342).
    // Fewer workgroups leave the row-block kernel ahead, whose pieces are finer.
    // bf16: 10 prompts of 23 tokens (104) 14.5 us against 13.8, of 70 (64) 14.6 against
    // 17.1, 15 of 27 (56) 9.4 against 13.7; fp32: 26 against 29 at 131, 39 against 35 at
    // 176; a few rows after thousands of tokens, whose keys are cut below, 105
    // against 50 at 64 (a table of 4096 tokens whose requests are short gives those
    // of 56 to 111 the slower side of the figures before).  (256 wide in fp32,
    // queries and output alone fill the registers.)
    pl.tiled = (groups >= (p.dtype == STAR_BF16 ? 112 : 160) || (groups >= 56 && keys >= 4096)) &&
               !(p.dtype == STAR_F32 && p.head_dim == 256);
    if (!pl.tiled) return;
    const int64_t most = tile_blocks(p.n_rows, g, p.n_seq);
    const int64_t key_tiles = keys / (p.head_dim * e > 256 ? 32 : 64);
    int splits = 1;
    pl.part_tiles = kPartTiles;
    if (2 * groups <= kPlaces) {
        // Places stay free: each block's keys are cut, into parts that pay from
        // sixteen tiles each (512 rows after 16000 tokens: 416 -> 172 us; after
        // 512, two parts of eight tiles: 38 -> 43)
        splits = (int)std::min<int64_t>(kMaxParts, kPlaces / groups);
    } else {
        // Cut keys fill the last round of places better, for 4% of a round a
        // cut; a round that leaves every CU one workgroup takes 0.62 of one.
        // Worth it for long parts (300 workgroups over 9200 tokens: 300 -> 225
        // us; 520: 464 -> 384; 700: 512 against 532; 640 over a window of 4096:
        // 205 against 229)
        pl.part_tiles = 40;
        auto cost = [&](int s) {
            const double rounds = (double)groups * s / kPlaces, last = rounds - (int)rounds;
            return ((int)rounds + (last > 0.5 ? 1.0 : last > 0.0 ? 0.62 : 0.0)) / s +
                   0.04 * (s - 1);
        };
        for (int s = 2; s <= 3; ++s)
            if (cost(s) < 0.93 * cost(1) && cost(s) < cost(splits)) splits = s;
    }
    // (no more than the most keys could use)
    if (most * p.n_kv_heads <= kMaxTickets)
        pl.splits = (int)std::max<int64_t>(1, std::min<int64_t>(splits, key_tiles / pl.part_tiles));
    // (and parts of blocks that are longer than others)
    pl.items = most * pl.splits;
    if (pl.splits > 1 && p.n_seq <= 64) pl.items += kMoreParts / p.n_kv_heads;
    pl.part_bytes = pl.splits == 1 ? 0
                                   : (size_t)(pl.items * p.n_kv_heads) * (p.head_dim / 2 + 4) *
                                         kThreads * sizeof(float);
}

hipError_t launch_attend_tiles(const AttendArgs& a, int dtype, int head_dim, hipStream_t stream) {
    return dtype == STAR_BF16 ? launch_tiles_of<STAR_BF16>(a, head_dim, stream)
                              : launch_tiles_of<STAR_F32>(a, head_dim, stream);
}

}  // namespace star
