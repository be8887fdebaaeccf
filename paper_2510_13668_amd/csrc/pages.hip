// Page tables of the key-value cache (include/star.h, "pages of the cache"):
// growth, release, forks, migrations and compaction, with the page copies they
// need.
//
// Both calls are two launches.  The first runs one workgroup per instance over
// the instance's reference counts and requests and decides everything: which
// free page goes where, who is served, what is copied.  The second carries it
// out: some workgroups write rows and reference counts, the others copy pages.
#include "star_common.hpp"
#include "star_internal.hpp"

namespace star {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kRunThreads = 256;

// What the first launch decides for one slot.
struct SlotPlan {
    int32_t from;       // the slot its first pages come from
    int32_t shared;     // pages taken over as they are
    int32_t kept;       // pages whose tokens it keeps: [shared, kept) are copied
    int32_t pages;      // pages of the new row
    int32_t old_pages;  // pages of the row before
    int32_t first;      // its first entry in the instance's list of free pages
    int32_t inst;       // the instance it is on afterwards
    int32_t served;     // 0: left as it was
};
static_assert(sizeof(SlotPlan) == kSlotPlanBytes, "workspace layout");

// Four counts of a wave's next 256 pages from page at, -1 past the end
// (the counts need no alignment beyond their own).
__device__ inline void load_counts(const int32_t* refs, int at, int end, int lane, int (&x)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int p = at + k * kWave + lane;
        x[k] = p < end ? refs[p] : -1;
    }
}

__device__ inline int lanes_below(uint64_t mask, int lane) {
    return __popcll(mask & ((1ull << lane) - 1));
}

struct AssignArgs {
    const int32_t *parent, *new_len, *inst_of, *table, *seq_len, *seq_inst, *refs;
    int32_t *table_out, *len_out, *inst_out, *refs_out;
    char* kv;
    SlotPlan* plan;
    int32_t* free_list;   // [n_inst][P]
    int32_t* copies;      // [n_inst][P][2] (source, target)
    int32_t* n_copies;    // [n_inst]
    int32_t* taken;       // [n_seq]: pages of a slot that forks share (cut slots alone)
    int32_t* err;
    int n_seq, max_pages, n_pages, n_inst, ps_log2, n_layers;
    int64_t page_bytes, page_stride, layer_stride;
};

// The counts that forks leave for the slots they share pages of are set, raised
// and read by one workgroup's threads, past the caches.
__device__ inline void taken_set(int32_t* x) {
    __hip_atomic_store(x, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline void taken_raise(int32_t* x, int pages) {
    __hip_atomic_fetch_max(x, pages, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline int taken_read(const int32_t* x) {
    return __hip_atomic_load(x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// One slot's demand, from its arrays, and where a cut slot keeps its last page
// (cut), from what forks of this call take of it (taken; null: nothing).
__device__ inline SlotPlan plan_slot(const AssignArgs& a, int b, const int32_t* taken, int& need,
                                     bool& cut, int32_t& bad) {
    SlotPlan s;
    const int ps = 1 << a.ps_log2, most = a.max_pages << a.ps_log2;
    const int len = a.seq_len[b], want = a.new_len[b];
    const int inst = a.seq_inst ? a.seq_inst[b] : 0;
    int to = a.inst_of ? a.inst_of[b] : inst;
    int from = a.parent ? a.parent[b] : b;
    bool ok = true;
    if (len < 0 || len > most || want < 0 || want > most) ok = false, bad |= STAR_DEV_BAD_LEN;
    if ((uint32_t)inst >= (uint32_t)a.n_inst || (uint32_t)to >= (uint32_t)a.n_inst)
        ok = false, bad |= STAR_DEV_BAD_INST;
    if (from < -1 || from >= a.n_seq) ok = false, bad |= STAR_DEV_BAD_PARENT;
    int keep = 0, shared = 0;
    cut = false;
    if (ok && from >= 0) {
        int from_len = len, from_inst = inst;
        if (from != b) {
            from_len = a.seq_len[from];
            from_inst = a.seq_inst ? a.seq_inst[from] : 0;
            if (from_len < 0 || from_len > most) ok = false, bad |= STAR_DEV_BAD_LEN;
            if ((uint32_t)from_inst >= (uint32_t)a.n_inst) ok = false, bad |= STAR_DEV_BAD_INST;
        }
        keep = min(want, ok ? from_len : 0);
        if (ok && from_inst == to) {
            // The page that the next tokens go into has to be the slot's alone, and
            // so has that of the last token where attention may store it anew before
            // the slot grows: after a cut, and in a fork
            const bool anew = from != b || want < from_len;
            shared = max(0, anew ? min(want - 1, from_len) : from_len) >> a.ps_log2;
            if (from == b && shared << a.ps_log2 < keep) {
                const int last = a.table[(int64_t)b * a.max_pages + shared];
                if ((uint32_t)last < (uint32_t)a.n_pages && a.refs[last] == 1) {
                    cut = anew;
                    if (!(cut && taken && taken_read(taken + b) > shared)) ++shared;
                }
            }
        }
    }
    s.from = from;
    s.shared = shared;
    s.kept = (keep + ps - 1) >> a.ps_log2;
    s.pages = ok ? (want + ps - 1) >> a.ps_log2 : 0;
    s.old_pages = len < 0 || len > most ? 0 : (len + ps - 1) >> a.ps_log2;
    s.inst = ok ? to : -1;
    s.first = 0;
    s.served = ok;
    need = ok ? s.pages - s.shared : 0;
    return s;
}

// A wave's stretch of an instance's P pages, a multiple of 256.
__device__ inline int stretch_of(int P) {
    return ((P + kPlanWaves - 1) / kPlanWaves + 255) / 256 * 256;
}

__global__ __launch_bounds__(kPlanThreads) void assign_plan_kernel(AssignArgs a) {
    __shared__ int s_count[kPlanWaves], s_copies;
    __shared__ bool s_cuts[kPlanWaves];
    __shared__ int64_t s_tmp[2 * kPlanWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int P = a.n_pages / a.n_inst;
    if (blockIdx.x >= (unsigned)a.n_inst) {
        // the other workgroups carry the counts over
        if (a.refs_out != a.refs)
            for (int64_t p = (int64_t)(blockIdx.x - a.n_inst) * kPlanThreads + tid; p < a.n_pages;
                 p += (int64_t)(gridDim.x - a.n_inst) * kPlanThreads)
                a.refs_out[p] = a.refs[p];
        return;
    }
    const int inst = blockIdx.x, page0 = inst * P;
    const int32_t* refs = a.refs + page0;
    if (tid == 0) s_copies = 0;

    // Everything that depends on arrays alone is asked for first: the first
    // stretch of counts, and this thread's first slot.
    const int stretch = stretch_of(P);
    const int from = min(P, wave * stretch), to = min(P, from + stretch);
    constexpr int kHeld = 2;                    // counts kept in registers: 512 a wave
    int held[kHeld][4];
#pragma unroll
    for (int h = 0; h < kHeld; ++h) load_counts(refs, from + 256 * h, to, lane, held[h]);
    const int per = (a.n_seq + kPlanThreads - 1) / kPlanThreads;
    const int b0 = min(a.n_seq, tid * per), b1 = min(a.n_seq, b0 + per);
    int32_t bad = 0;
    int need0 = 0;
    SlotPlan slot0 = {};
    slot0.inst = -1;
    int64_t mine = 0, copying = 0;
    const int32_t* taken = nullptr;
    bool cuts = false, cut;
    auto demands = [&]() {
        mine = copying = 0;
        for (int b = b0; b < b1; ++b) {
            int need;
            const SlotPlan s = plan_slot(a, b, taken, need, cut, bad);
            if (b == b0) slot0 = s, need0 = need;
            if (s.inst == inst) mine += need, copying += s.kept - s.shared, cuts |= cut;
        }
    };
    demands();

    // the instance's free pages in order: each wave counts its stretch, then
    // writes it behind the waves before
    int n = 0;
    for (int at = from, h = 0; at < to; at += 256, ++h) {
        int x[4];
        if (h >= kHeld) load_counts(refs, at, to, lane, x);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            n += __popcll(__ballot((h == 0 ? held[0][k] : h == 1 ? held[1][k] : x[k]) == 0));
    }
    const bool cuts_here = __any(cuts);
    if (lane == 0) s_count[wave] = n, s_cuts[wave] = cuts_here;
    int64_t upto, k;
    auto running = [&]() {
        upto = mine, k = copying;
        block_incl_add2_i64<kPlanThreads>(upto, k, s_tmp);
        upto -= mine, k -= copying;
    };
    running();
    int n_free = 0, rank = 0;
    bool any_cuts = false;
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) rank += s_count[w];
        n_free += s_count[w];
        any_cuts |= s_cuts[w];
    }
    if (a.parent && any_cuts) {
        // a cut slot's last page may be one that a fork takes as a full one: the
        // forks say how many pages they share before the demands count
        for (int b = b0; b < b1; ++b) {
            int need;
            if (plan_slot(a, b, nullptr, need, cut, bad).inst == inst && cut)
                taken_set(a.taken + b);
        }
        xch_wait_stores();
        __syncthreads();
        for (int b = b0; b < b1; ++b) {
            int need;
            const SlotPlan s = plan_slot(a, b, nullptr, need, cut, bad);
            if (s.inst == inst && s.from >= 0 && s.from != b && s.shared)
                taken_raise(a.taken + s.from, s.shared);
        }
        xch_wait_stores();
        __syncthreads();
        taken = a.taken;
        demands();
        running();
    }
    int32_t* list = a.free_list + page0;
    for (int at = from, h = 0; at < to; at += 256, ++h) {
        int x[4];
        if (h >= kHeld) load_counts(refs, at, to, lane, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool free = (h == 0 ? held[0][j] : h == 1 ? held[1][j] : x[j]) == 0;
            const uint64_t mask = __ballot(free);
            if (free) list[rank + lanes_below(mask, lane)] = page0 + at + j * kWave + lane;
            rank += __popcll(mask);
        }
    }
    __syncthreads();           // the list is written (the copies read it)

    // Its slots in order take them.  Running demands only grow, so the slots
    // served come before all those that are not: their running counts of
    // copies need no second pass
    int last_copy = 0;
    for (int i = 0; i < per; ++i) {
        const int b = b0 + i;
        int copies = 0;
        SlotPlan s = slot0;
        if (b < b1) {
            int need = need0;
            if (i > 0) s = plan_slot(a, b, taken, need, cut, bad);
            if (s.inst == inst) {
                s.first = (int)min(upto, (int64_t)P);
                upto += need;
                if (need > 0 && upto > n_free) s.served = 0, bad |= STAR_DEV_NO_PAGES;
                if (s.served) copies = s.kept - s.shared;
            }
            if (s.inst == inst || (s.inst < 0 && inst == 0)) a.plan[b] = s;
        }
        // A slot's copies go on the list: a few (a fork's last page) by its own
        // thread, more by its wave, 64 pages at once
        constexpr int kFew = 4;
        if (copies > 0 && copies <= kFew) {
            const int32_t* row = a.table + (int64_t)s.from * a.max_pages + s.shared;
            for (int j = 0; j < copies; ++j) {
                int src = row[j];
                if ((uint32_t)src >= (uint32_t)a.n_pages) src = -1, bad |= STAR_DEV_BAD_PAGE;
                a.copies[2 * (page0 + k + j)] = src;
                a.copies[2 * (page0 + k + j) + 1] = list[s.first + j];
            }
        }
        for (uint64_t todo = __ballot(copies > kFew); todo; todo &= todo - 1) {
            const int x = __builtin_ctzll(todo);
            const int count = __builtin_amdgcn_readlane(copies, x);
            const int shared = __builtin_amdgcn_readlane(s.shared, x);
            const int first = __builtin_amdgcn_readlane(s.first, x);
            const int at = __builtin_amdgcn_readlane((int)k, x);
            const int32_t* row =
                a.table + (int64_t)__builtin_amdgcn_readlane(s.from, x) * a.max_pages + shared;
            for (int j = lane; j < count; j += kWave) {
                int src = row[j];
                if ((uint32_t)src >= (uint32_t)a.n_pages) src = -1, bad |= STAR_DEV_BAD_PAGE;
                a.copies[2 * (page0 + at + j)] = src;
                a.copies[2 * (page0 + at + j) + 1] = list[first + j];
            }
        }
        k += copies;
        if (copies) last_copy = (int)k;
    }
    if (last_copy) atomicMax(&s_copies, last_copy);
    __syncthreads();
    if (tid == 0) a.n_copies[inst] = s_copies;
    report_error(a.err, bad);
}

// Page copies: source and target pages of every instance's list, in all
// layers, kLanes threads a page and layer; 16 bytes a thread and load, eight
// loads in flight.  Nothing copied is read again here, so it passes the caches
// by (2048 pages of 28 layers compacted: 188 -> 182 us; migrations 74 -> 69).
template <int kLanes>
__device__ inline void copy_pages_by(char* kv, const int32_t* copies, const int32_t* n_copies,
                                     int n_inst, int P, int n_layers, int64_t page_bytes,
                                     int64_t page_stride, int64_t layer_stride, int worker,
                                     int workers) {
    constexpr int kTeams = kRunThreads / kLanes;
    int64_t item = (int64_t)worker * kTeams + threadIdx.x / kLanes, base = 0;
    for (int i = 0; i < n_inst; ++i) {
        const int64_t n = (int64_t)n_copies[i] * n_layers;
        for (; item < base + n; item += (int64_t)workers * kTeams) {
            const int64_t x = item - base;
            const int64_t k = (x >> 32 ? x / n_layers : (uint32_t)x / (uint32_t)n_layers);
            const int layer = (int)(x - k * n_layers);
            const u32x2 pair = *(const u32x2*)(copies + 2 * (k + (int64_t)i * P));
            const int src = (int)pair[0], dst = (int)pair[1];
            if (src < 0) continue;
            const char* from = kv + layer * layer_stride + src * page_stride;
            char* to = kv + layer * layer_stride + dst * page_stride;
            constexpr int kStep = kLanes * 16, kUnroll = 8;
            int64_t at = threadIdx.x % kLanes * 16;
            for (; at + (kUnroll - 1) * kStep < page_bytes; at += kUnroll * kStep) {
                u32x4 v[kUnroll];
#pragma unroll
                for (int q = 0; q < kUnroll; ++q)
                    v[q] = __builtin_nontemporal_load((const u32x4*)(from + at + q * kStep));
#pragma unroll
                for (int q = 0; q < kUnroll; ++q)
                    __builtin_nontemporal_store(v[q], (u32x4*)(to + at + q * kStep));
            }
            for (; at < page_bytes; at += kStep)
                __builtin_nontemporal_store(__builtin_nontemporal_load((const u32x4*)(from + at)),
                                            (u32x4*)(to + at));
        }
        base += n;
    }
}
// A small page is a few lanes' or a wave's, so that many are in flight: each
// waits for its place in the list first (1440-byte pages: 147 -> 69 us).
__device__ inline void copy_pages(char* kv, const int32_t* copies, const int32_t* n_copies,
                                  int n_inst, int P, int n_layers, int64_t page_bytes,
                                  int64_t page_stride, int64_t layer_stride, int worker,
                                  int workers) {
    if (page_bytes <= 512)
        copy_pages_by<8>(kv, copies, n_copies, n_inst, P, n_layers, page_bytes, page_stride,
                         layer_stride, worker, workers);
    else if (page_bytes <= 8192)
        copy_pages_by<64>(kv, copies, n_copies, n_inst, P, n_layers, page_bytes, page_stride,
                          layer_stride, worker, workers);
    else
        copy_pages_by<256>(kv, copies, n_copies, n_inst, P, n_layers, page_bytes, page_stride,
                           layer_stride, worker, workers);
}

__global__ __launch_bounds__(kRunThreads) void assign_run_kernel(AssignArgs a, int row_groups) {
    const int P = a.n_pages / a.n_inst;
    if (blockIdx.x >= (unsigned)row_groups) {
        copy_pages(a.kv, a.copies, a.n_copies, a.n_inst, P, a.n_layers, a.page_bytes,
                   a.page_stride, a.layer_stride, blockIdx.x - row_groups,
                   gridDim.x - row_groups);
        return;
    }
    // one wave a slot: its new row, and the counts of what comes and goes
    const int lane = threadIdx.x & (kWave - 1);
    int32_t bad = 0;
    for (int b = blockIdx.x * (kRunThreads / kWave) + threadIdx.x / kWave; b < a.n_seq;
         b += row_groups * (kRunThreads / kWave)) {
        const SlotPlan s = a.plan[b];
        const int32_t* old = a.table + (int64_t)b * a.max_pages;
        const int32_t* src = s.from >= 0 ? a.table + (int64_t)s.from * a.max_pages : old;
        int32_t* out = a.table_out + (int64_t)b * a.max_pages;
        if (lane == 0) {
            a.len_out[b] = s.served ? a.new_len[b] : a.seq_len[b];
            if (a.inst_out) a.inst_out[b] = s.served ? s.inst : a.seq_inst ? a.seq_inst[b] : 0;
        }
        if (!s.served) {
            for (int j = lane; j < s.old_pages; j += kWave) out[j] = old[j];
            continue;
        }
        const int32_t* list = a.free_list + (int64_t)s.inst * P + s.first;
        const bool stays = s.from == b;     // shared pages are its own already
        for (int j = lane; j < max(s.pages, s.old_pages); j += kWave) {
            const int was = j < s.old_pages ? old[j] : -1;
            if (j < s.old_pages && !(stays && j < s.shared)) {
                if ((uint32_t)was < (uint32_t)a.n_pages) atomicSub(a.refs_out + was, 1);
                else bad |= STAR_DEV_BAD_PAGE;
            }
            if (j >= s.pages) continue;
            const int page = j >= s.shared ? list[j - s.shared] : stays ? was : src[j];
            out[j] = page;
            if (!(stays && j < s.shared)) {
                if ((uint32_t)page < (uint32_t)a.n_pages) atomicAdd(a.refs_out + page, 1);
                else bad |= STAR_DEV_BAD_PAGE;
            }
        }
    }
    report_error(a.err, bad);
}

struct CompactArgs {
    const int32_t *table, *seq_len, *refs;
    int32_t *table_out, *refs_out, *n_live;
    char* kv;
    int32_t* map;        // [n_pages]: where each page's content goes
    int32_t* copies;     // [n_inst][P][2]
    int32_t* n_copies;   // [n_inst]
    int32_t* err;
    int n_seq, max_pages, n_pages, n_inst, ps_log2, n_layers;
    int64_t page_bytes, page_stride, layer_stride;
};

__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(CompactArgs a) {
    __shared__ int s_count[kPlanWaves], s_hole[kPlanWaves], s_high[kPlanWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int P = a.n_pages / a.n_inst, inst = blockIdx.x, page0 = inst * P;
    const int32_t* refs = a.refs + page0;
    const int stretch = stretch_of(P);
    const int from = min(P, wave * stretch), to = min(P, from + stretch);
    int n = 0;
    for (int at = from; at < to; at += 256) {
        int x[4];
        load_counts(refs, at, to, lane, x);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            n += __popcll(__ballot(x[k] != 0 && at + k * kWave + lane < to));
    }
    if (lane == 0) s_count[wave] = n;
    __syncthreads();
    int n_live = 0;
    for (int w = 0; w < kPlanWaves; ++w) n_live += s_count[w];
    // holes below n_live and live pages from there on, of each stretch
    int holes = 0, high = 0;
    for (int at = from; at < to; at += 256) {
        int x[4];
        load_counts(refs, at, to, lane, x);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int p = at + k * kWave + lane;
            holes += __popcll(__ballot(p < to && p < n_live && x[k] == 0));
            high += __popcll(__ballot(p < to && p >= n_live && x[k] != 0));
        }
    }
    if (lane == 0) s_hole[wave] = holes, s_high[wave] = high;
    __syncthreads();
    int hole = 0, up = 0, all = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) hole += s_hole[w], up += s_high[w];
        all += s_high[w];
    }
    // the i-th hole and the i-th high page meet in the list of copies
    int32_t* copies = a.copies + 2 * (int64_t)page0;
    for (int at = from; at < to; at += 256) {
        int x[4];
        load_counts(refs, at, to, lane, x);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int p = at + k * kWave + lane;
            const bool is_hole = p < to && p < n_live && x[k] == 0;
            const bool is_high = p < to && p >= n_live && x[k] != 0;
            const uint64_t mh = __ballot(is_hole), mu = __ballot(is_high);
            if (is_hole) copies[2 * (hole + lanes_below(mh, lane)) + 1] = page0 + p;
            if (is_high) copies[2 * (up + lanes_below(mu, lane))] = page0 + p;
            hole += __popcll(mh);
            up += __popcll(mu);
            if (p < to && !is_hole) a.refs_out[page0 + p] = is_high ? 0 : x[k];
            if (p < to && !is_high) a.map[page0 + p] = page0 + p;
        }
    }
    __syncthreads();
    for (int k = tid; k < all; k += kPlanThreads) {
        const int src = copies[2 * k], dst = copies[2 * k + 1];
        a.map[src] = dst;
        a.refs_out[dst] = a.refs[src];
    }
    if (tid == 0) {
        a.n_copies[inst] = all;
        a.n_live[inst] = n_live;
    }
}

__global__ __launch_bounds__(kRunThreads) void compact_run_kernel(CompactArgs a, int row_groups) {
    if (blockIdx.x >= (unsigned)row_groups) {
        copy_pages(a.kv, a.copies, a.n_copies, a.n_inst, a.n_pages / a.n_inst, a.n_layers,
                   a.page_bytes, a.page_stride, a.layer_stride, blockIdx.x - row_groups,
                   gridDim.x - row_groups);
        return;
    }
    const int lane = threadIdx.x & (kWave - 1), ps = 1 << a.ps_log2;
    int32_t bad = 0;
    for (int b = blockIdx.x * (kRunThreads / kWave) + threadIdx.x / kWave; b < a.n_seq;
         b += row_groups * (kRunThreads / kWave)) {
        const int len = a.seq_len[b];
        if (len < 0 || len > a.max_pages << a.ps_log2) {
            bad |= STAR_DEV_BAD_LEN;
            continue;
        }
        const int pages = (len + ps - 1) >> a.ps_log2;
        for (int j = lane; j < pages; j += kWave) {
            const int64_t at = (int64_t)b * a.max_pages + j;
            const int page = a.table[at];
            const bool ok = (uint32_t)page < (uint32_t)a.n_pages;
            if (!ok) bad |= STAR_DEV_BAD_PAGE;
            a.table_out[at] = ok ? a.map[page] : page;
        }
    }
    report_error(a.err, bad);
}

int row_groups_of(int n_seq) {
    const int g = (n_seq + kRunThreads / kWave - 1) / (kRunThreads / kWave);
    return g < 1 ? 1 : g < 1024 ? g : 1024;
}
// workgroups that copy: four a CU
constexpr int kCopyGroups = 1024;

}  // namespace

PagesPlan plan_pages(const star_pages_params& p) {
    PagesPlan pl;
    size_t at = STAR_WS_HEADER_BYTES;
    auto take = [&](size_t bytes) {
        const size_t x = at;
        at += align_up(bytes, 256);
        return x;
    };
    pl.n_copies_off = take((size_t)p.n_inst * 4);
    pl.copies_off = take((size_t)p.n_pages * 8);
    pl.list_off = take((size_t)p.n_pages * 4);           // free pages, or the page map
    pl.slots_off = take((size_t)p.n_seq * kSlotPlanBytes);
    pl.taken_off = take((size_t)p.n_seq * 4);
    pl.total = at;
    return pl;
}

hipError_t launch_assign(const star_pages_params& p, const PagesPlan& pl, const int32_t* parent,
                         const int32_t* new_len, const int32_t* inst_of, const int32_t* table,
                         const int32_t* seq_len, const int32_t* seq_inst, const int32_t* refs,
                         void* kv, int32_t* table_out, int32_t* len_out, int32_t* inst_out,
                         int32_t* refs_out, char* ws, hipStream_t stream) {
    AssignArgs a;
    a.parent = parent, a.new_len = new_len, a.inst_of = inst_of, a.table = table;
    a.seq_len = seq_len, a.seq_inst = seq_inst, a.refs = refs;
    a.table_out = table_out, a.len_out = len_out, a.inst_out = inst_out, a.refs_out = refs_out;
    a.kv = (char*)kv;
    a.plan = (SlotPlan*)(ws + pl.slots_off);
    a.free_list = (int32_t*)(ws + pl.list_off);
    a.copies = (int32_t*)(ws + pl.copies_off);
    a.n_copies = (int32_t*)(ws + pl.n_copies_off);
    a.taken = (int32_t*)(ws + pl.taken_off);
    a.err = (int32_t*)(ws + kHdrErrorWord);
    a.n_seq = p.n_seq, a.max_pages = p.max_pages, a.n_pages = p.n_pages, a.n_inst = p.n_inst;
    a.ps_log2 = __builtin_ctz(p.page_size), a.n_layers = p.n_layers;
    a.page_bytes = p.page_bytes, a.page_stride = p.page_stride, a.layer_stride = p.layer_stride;
    int carry = (p.n_pages + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
    carry = refs_out == refs ? 0 : carry < 256 ? carry : 256;
    hipLaunchKernelGGL(assign_plan_kernel, dim3(p.n_inst + carry), dim3(kPlanThreads), 0, stream,
                       a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int rows = row_groups_of(p.n_seq);
    hipLaunchKernelGGL(assign_run_kernel, dim3(rows + kCopyGroups), dim3(kRunThreads), 0, stream,
                       a, rows);
    return hipGetLastError();
}

hipError_t launch_compact(const star_pages_params& p, const PagesPlan& pl, const int32_t* table,
                          const int32_t* seq_len, const int32_t* refs, void* kv,
                          int32_t* table_out, int32_t* refs_out, int32_t* n_live, char* ws,
                          hipStream_t stream) {
    CompactArgs a;
    a.table = table, a.seq_len = seq_len, a.refs = refs;
    a.table_out = table_out, a.refs_out = refs_out, a.n_live = n_live;
    a.kv = (char*)kv;
    a.map = (int32_t*)(ws + pl.list_off);
    a.copies = (int32_t*)(ws + pl.copies_off);
    a.n_copies = (int32_t*)(ws + pl.n_copies_off);
    a.err = (int32_t*)(ws + kHdrErrorWord);
    a.n_seq = p.n_seq, a.max_pages = p.max_pages, a.n_pages = p.n_pages, a.n_inst = p.n_inst;
    a.ps_log2 = __builtin_ctz(p.page_size), a.n_layers = p.n_layers;
    a.page_bytes = p.page_bytes, a.page_stride = p.page_stride, a.layer_stride = p.layer_stride;
    hipLaunchKernelGGL(compact_plan_kernel, dim3(p.n_inst), dim3(kPlanThreads), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int rows = row_groups_of(p.n_seq);
    hipLaunchKernelGGL(compact_run_kernel, dim3(rows + kCopyGroups), dim3(kRunThreads), 0, stream,
                       a, rows);
    return hipGetLastError();
}

}  // namespace star
