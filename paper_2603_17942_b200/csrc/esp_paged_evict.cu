// Cutting caches to their budgets, and the acceptance of draft trees: the two operators that move slots of a paged cache.
//
// Eviction: a list of a sequence and KV head is a choice of its `budget` largest keys (score, recency), 32-bit numbers in the order of
// the scores.  k_evict_select, a block or a cluster of blocks for each list, finds the smallest key that stays by its digits, four times eight bits, with histograms in shared memory,
// then deals the kept slots behind the budget to the dropped ones in front of it, both in order, so the answer depends on nothing but the numbers.
// k_evict_move moves the lists' rows, scores and positions, spread over the whole GPU.  Both are chains of short steps: what counts is that the loads of a step are all under
// way before the first is waited for, and that the code is short (loops unrolled over 32 keys in registers took longer to fetch than to run).
// Clusters with the keys in shared memory, and the last two digits from the keys themselves where few share the first two, took 8 sequences of 32k positions cut to 4k, 8 heads of
// 128, from 121 to 78 us: 28 for the choice and 50 for 235 MB of rows, at 0.73 of the copy rate.  32 sequences that are one position above their budget: 14 us, 42 with table and scratch for 64k positions (seven blocks of eight that leave at once).
#include <cooperative_groups.h>

#include "esp_paged.cuh"

namespace cg = cooperative_groups;

namespace esp {

namespace {

using namespace paged;

__device__ __forceinline__ size_t slot_offset(const SlotsView& v, int page, int slot, int head) {
    return (size_t)((long long)page * v.page + (long long)slot * v.tok + (long long)head * v.head);
}
__device__ __forceinline__ size_t row_offset(const PagesView& v, int page, int slot, int head) {
    return (size_t)((long long)page * v.page + (long long)slot * v.tok + (long long)head * v.head);
}

// The table's entry, whatever it says, and the page it names or -1: several loads can be under way before the first is looked at (load_page branches on each)
__device__ __forceinline__ int table_entry(const SeqTable& t, int b, int index) { return __ldg(t.table + (size_t)b * t.table_stride + index); }
__device__ __forceinline__ int named(const PagesView& p, int entry) { return entry >= 0 && entry < p.n_pages ? entry : -1; }

// Larger numbers for larger scores, equal ones for equal scores (-0 = 0); a NaN as -infinity.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) x = -INFINITY;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t KEY_INF = 0xff800000u;      // order_key(INFINITY)

constexpr int BINS = 256, MAX_CL = EVICT_BLOCKS, NEAR = 255;
constexpr int KEYS = EVICT_KEYS;      // keys that a block keeps; those of a longer stretch are made anew in every pass

struct SeqCut {
    int kv, budget;
    int settled, base;    // slots in front of `settled` have a position of their own, slot s behind them has base + s
    bool cut;
};
__device__ __forceinline__ SeqCut load_cut(const EvictArgs& a, int b) {
    SeqCut c;
    c.kv = __ldg(a.seq.kv_len + b);
    c.budget = __ldg(a.budget + b);
    c.base = a.positions.p ? __ldg(a.seen + b) - c.kv : 0;
    c.settled = a.positions.p ? a.settled[b] : 0;
    c.cut = false;
    if (c.kv < 0 || c.kv > a.seq.kv_cap || c.budget < 0) set_error(a.seq.status, DEV_E_INDEX);
    else if (c.kv > c.budget) {
        if (c.budget < a.recent) set_error(a.seq.status, DEV_E_INDEX);
        else if (c.kv / 2 > a.list_cap) set_error(a.seq.status, DEV_E_CAPACITY);
        else c.cut = true;
    }
    return c;
}
// Row of `bytes` bytes, VEC of them to a lane
template <int VEC> struct Unit;
template <> struct Unit<16> { typedef uint4 T; };
template <> struct Unit<8> { typedef uint2 T; };
template <> struct Unit<4> { typedef uint32_t T; };
template <> struct Unit<2> { typedef uint16_t T; };

// One move by a warp: keys, values, score and position.  settled, base: what slots hold as positions, as in SeqCut.
template <int VEC>
__device__ __forceinline__ void move_one(const EvictArgs& a, int elem, int b, int h, const SeqCut& c, int2 x, int lane) {
    typedef typename Unit<VEC>::T U;
    const int row = a.D * elem / VEC, fi = page_index(a.pages, x.x), ti = page_index(a.pages, x.y), fs = x.x - fi * a.pages.page_size, ts = x.y - ti * a.pages.page_size;
    int fp = table_entry(a.seq, b, fi), tp = table_entry(a.seq, b, ti);
    fp = named(a.pages, fp);
    tp = named(a.pages, tp);
    if (fp < 0 || tp < 0) {
        set_error(a.seq.status, DEV_E_INDEX);
        return;
    }
    for (int u = lane; u < 2 * row; u += 32) {
        char* base = reinterpret_cast<char*>(u < row ? a.pages.k : a.pages.v) + (size_t)(u < row ? u : u - row) * VEC;
        *reinterpret_cast<U*>(base + row_offset(a.pages, tp, ts, h) * elem) = *reinterpret_cast<const U*>(base + row_offset(a.pages, fp, fs, h) * elem);
    }
    if (lane == 0) {
        reinterpret_cast<float*>(a.scores.p)[slot_offset(a.scores, tp, ts, h)] = reinterpret_cast<const float*>(a.scores.p)[slot_offset(a.scores, fp, fs, h)];
        if (a.positions.p)
            reinterpret_cast<int32_t*>(a.positions.p)[slot_offset(a.positions, tp, ts, h)] =
                x.x < c.settled ? reinterpret_cast<const int32_t*>(a.positions.p)[slot_offset(a.positions, fp, fs, h)] : c.base + x.x;
    }
}

// The keys of slots first + step * j below `end`, j < N, 0 for the others (no key of a slot is 0): all pages first, then all scores and positions, so that the loads wait for each other
// twice and not 2 N times.
template <int N>
__device__ __forceinline__ void load_keys(const EvictArgs& a, const SeqCut& c, int b, int h, int first, int step, int end, uint32_t (&k)[N]) {
    int page[N], slot[N];
    float x[N];
    bool bad = false;
    const float* scores = reinterpret_cast<const float*>(a.scores.p) + (long long)h * a.scores.head;
    const int32_t* positions = reinterpret_cast<const int32_t*>(a.positions.p) + (a.positions.p ? (long long)h * a.positions.head : 0);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int s = min(first + step * j, c.kv - 1), index = page_index(a.pages, s);
        page[j] = table_entry(a.seq, b, index);
        slot[j] = s - index * a.pages.page_size;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        page[j] = named(a.pages, page[j]);
        bad = bad || (page[j] < 0 && first + step * j < end);
    }
    if (bad) set_error(a.seq.status, DEV_E_INDEX);
#pragma unroll
    for (int j = 0; j < N; ++j)
        x[j] = page[j] < 0 ? -INFINITY : scores[page[j] * a.scores.page + slot[j] * a.scores.tok];
    int pos[N];
#pragma unroll
    for (int j = 0; j < N; ++j) pos[j] = c.base + first + step * j;
    if (a.positions.p && a.recent > 0) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (first + step * j < c.settled) pos[j] = page[j] < 0 ? -1 : positions[page[j] * a.positions.page + slot[j] * a.positions.tok];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        k[j] = order_key(x[j]);
        // (positions differ, so they are told apart in 64 bits)
        if (a.recent > 0 && (long long)pos[j] >= (long long)c.base + c.kv - a.recent) k[j] = KEY_INF;
        if (first + step * j >= end) k[j] = 0;
    }
}

constexpr int SELECT_THREADS = 512;
template <int VEC>
__global__ void __launch_bounds__(SELECT_THREADS) k_evict_select(const __grid_constant__ EvictArgs a, int elem) {
    constexpr int THREADS = SELECT_THREADS, WARPS = THREADS / 32;
    __shared__ uint32_t s_key[KEYS];
    __shared__ uint32_t s_hist[2][BINS];                // (a block of the cluster may be a digit ahead of another)
    __shared__ int s_all[BINS];
    __shared__ int s_warp[WARPS], s_warp2[WARPS], s_word[4];
    __shared__ int2 s_count[MAX_CL];                    // [block] (kept ones behind the budget, dropped ones in front of it)
    __shared__ int s_ties[MAX_CL];
    __shared__ uint32_t s_near[MAX_CL][NEAR + 1];       // [block] the keys that share the digits found so far; the last one: how many
    __shared__ int s_near_n;
    cg::cluster_group cluster = cg::this_cluster();
    int CL = cluster.num_blocks();
    const int me = cluster.block_rank(), list_no = blockIdx.x / CL;
    const int b = list_no / a.Hkv, h = list_no - b * a.Hkv, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t low = (1u << lane) - 1u;
    pdl_launch_dependents();
    const SeqCut c = load_cut(a, b);
    if (!c.cut) {                                       // the same in the whole cluster
        if (me == 0 && threadIdx.x == 0) {
            a.count[list_no] = 0;
            if (h == 0) a.info[b] = make_int4(-1, 0, 0, 0);
        }
        return;
    }
    if (a.as_needed && c.kv <= KEYS) {                  // the first block has the list alone (and nothing to do with the others)
        if (me != 0) return;
        CL = 1;
    }
    if (CL > 1) cluster.barrier_arrive();               // (before anybody looks into another block's shared memory, all have to have started)
    // the block's stretch of slots, and each warp's of it
    const int per = (c.kv + CL * 32 - 1) / (CL * 32) * 32, f0 = min(c.kv, me * per), f1 = min(c.kv, f0 + per);
    const int each = (per + THREADS - 1) / THREADS * 32, s0 = min(f1, f0 + warp * each), s1 = min(f1, s0 + each);
    const bool kept = per <= KEYS;
    if (kept) {
        constexpr int N = 4;
#pragma unroll 1
        for (int i = f0 + (int)threadIdx.x; i < f1; i += N * THREADS) {
            uint32_t k[N];
            load_keys<N>(a, c, b, h, i, THREADS, f1, k);
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (i + j * THREADS < f1) s_key[i + j * THREADS - f0] = k[j];
        }
    }
    // f(slot of this lane, its key) over the warp's stretch, by all lanes together
    auto walk = [&](auto f) {
        if (kept) {
#pragma unroll 2
            for (int i = s0 + lane; i - lane < s1; i += 32) f(i, i < s1 ? s_key[i - f0] : 0u);
        } else {
            constexpr int N = 4;
            for (int i = s0 + lane; i - lane < s1; i += 32 * N) {
                uint32_t k[N];
                load_keys<N>(a, c, b, h, i, 32, s1, k);
#pragma unroll
                for (int j = 0; j < N; ++j) f(i + 32 * j, k[j]);
            }
        }
    };
    auto before = [&](const int* of) { return (int)__reduce_add_sync(0xffffffffu, lane < warp && lane < WARPS ? of[lane] : 0); };     // the sum over the warps in front
    if (CL > 1) cluster.barrier_wait();

    // ---- the smallest key that stays, `top`, how many keys are above it, and how many equal it
    uint32_t top = 0, mask = 0;
    int above = 0, same = 0;
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (shift == 8 && c.budget > 0) {
            // few keys share two digits, as a rule: everybody gets all of them, and each counts those above it
            if (threadIdx.x == 0) s_near_n = 0;
            __syncthreads();
            walk([&](int, uint32_t k) {
                if (k != 0 && (k & mask) == top) {
                    const int i = atomicAdd(&s_near_n, 1);
                    if (i < NEAR)
                        for (int r = 0; r < CL; ++r) cluster.map_shared_rank(&s_near[0][0], r)[me * (NEAR + 1) + i] = k;
                }
            });
            __syncthreads();
            if ((int)threadIdx.x < CL) cluster.map_shared_rank(&s_near[0][0], threadIdx.x)[me * (NEAR + 1) + NEAR] = (uint32_t)s_near_n;
            if (CL > 1) cluster.sync();
            else __syncthreads();
            bool fits = true;
#pragma unroll
            for (int r = 0; r < MAX_CL; ++r) fits = fits && (r >= CL || s_near[r][NEAR] <= NEAR);
            if (fits) {
                for (int i = threadIdx.x; i < CL * NEAR; i += THREADS) {
                    const int r = i / NEAR, e = i % NEAR;
                    if (e >= (int)s_near[r][NEAR]) continue;
                    const uint32_t k = s_near[r][e];
                    int over = above, eq = 0;
                    for (int q = 0; q < CL; ++q) {
                        const int n = (int)s_near[q][NEAR];
#pragma unroll 4
                        for (int j = 0; j < n; ++j) {
                            over += s_near[q][j] > k;
                            eq += s_near[q][j] == k;
                        }
                    }
                    if (over < c.budget && c.budget <= over + eq) {      // (equal ones all write the same)
                        s_word[0] = (int)k;
                        s_word[1] = over;
                        s_word[2] = eq;
                    }
                }
                __syncthreads();
                top = (uint32_t)s_word[0];
                above = s_word[1];
                same = s_word[2];
                break;
            }
        }
        uint32_t* hist = s_hist[(shift >> 3) & 1];
        for (int i = threadIdx.x; i < BINS; i += THREADS) hist[i] = 0;
        __syncthreads();
        walk([&](int, uint32_t k) {
            if (k != 0 && (k & mask) == top) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        });
        if (CL > 1) cluster.sync();
        else __syncthreads();
        if (threadIdx.x < BINS) {
            int n = 0;
            if (CL == 1) n = (int)hist[threadIdx.x];
            else {
                uint32_t part[MAX_CL];
#pragma unroll
                for (int r = 0; r < MAX_CL; ++r) part[r] = r < CL ? cluster.map_shared_rank(hist, r)[threadIdx.x] : 0u;
#pragma unroll
                for (int r = 0; r < MAX_CL; ++r) n += (int)part[r];
            }
            s_all[threadIdx.x] = n;
        }
        __syncthreads();
        if (warp == 0) {                                // bins from the top, eight of them to a lane
            int n[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] = s_all[BINS - 1 - 8 * lane - i];
                sum += n[i];
            }
            int front = above + (int)warp_scan_u32(sum, lane) - sum;
            if (lane == 0 && c.budget == 0) { s_word[0] = BINS - 1; s_word[1] = s_word[2] = 0; }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (front < c.budget && c.budget <= front + n[i]) {
                    s_word[0] = BINS - 1 - 8 * lane - i;
                    s_word[1] = front;
                    s_word[2] = n[i];
                }
                front += n[i];
            }
        }
        __syncthreads();
        above = s_word[1];
        same = s_word[2];
        top |= (uint32_t)s_word[0] << shift;
        mask |= 255u << shift;
    }
    const int ties = c.budget - above;                  // slots with the key `top` that stay: the first ones of `same`

    // ---- kept ones behind the budget and dropped ones in front of it, in order
    const bool some = ties < same;                      // which of the equal ones is a matter of order
    int tie = 0;
    if (some) {
        int n = 0;
        walk([&](int, uint32_t k) { n += __popc(__ballot_sync(0xffffffffu, k == top)); });
        if (lane == 0) s_warp[warp] = n;
        __syncthreads();
        tie = before(s_warp);
        if (CL > 1) {
            if (warp == WARPS - 1 && lane < CL) cluster.map_shared_rank(s_ties, lane)[me] = tie + n;
            cluster.sync();
            for (int r = 0; r < me; ++r) tie += s_ties[r];
        }
        __syncthreads();
    }
    const int tie0 = tie;
    auto stays = [&](uint32_t k) {                      // all lanes
        if (!some) return k >= top && k != 0;
        const uint32_t eq = __ballot_sync(0xffffffffu, k == top);
        const bool s = k > top || (k == top && tie + __popc(eq & low) < ties);
        tie += __popc(eq);
        return s;
    };
    int go = 0, to = 0;
    walk([&](int s, uint32_t k) {
        const bool st = stays(k);
        go += __popc(__ballot_sync(0xffffffffu, st && s >= c.budget));
        to += __popc(__ballot_sync(0xffffffffu, k != 0 && !st && s < c.budget));
    });
    if (lane == 0) { s_warp[warp] = go; s_warp2[warp] = to; }
    __syncthreads();
    int m = before(s_warp), e = before(s_warp2), total;
    if (CL > 1) {
        if (warp == WARPS - 1 && lane < CL) cluster.map_shared_rank(s_count, lane)[me] = make_int2(m + go, e + to);
        cluster.sync();
        total = 0;
        for (int r = 0; r < CL; ++r) {
            const int2 x = s_count[r];
            if (r < me) { m += x.x; e += x.y; }
            total += x.x;
        }
    } else {
        total = (int)__reduce_add_sync(0xffffffffu, lane < WARPS ? s_warp[lane] : 0);
    }
    int2* list = a.list + (size_t)list_no * a.list_cap;
    tie = tie0;
    if (total > 0)
        walk([&](int s, uint32_t k) {
            const bool st = stays(k);
            const uint32_t gm = __ballot_sync(0xffffffffu, st && s >= c.budget), tm = __ballot_sync(0xffffffffu, k != 0 && !st && s < c.budget);
            const int mi = m + __popc(gm & low), ei = e + __popc(tm & low);      // (pages that are not the sequence's own may have changed since they were counted)
            if (((gm >> lane) & 1) && mi < a.list_cap) list[mi].x = s;
            if (((tm >> lane) & 1) && ei < a.list_cap) list[ei].y = s;
            m += __popc(gm);
            e += __popc(tm);
        });
    // few moves of a list that one block has are made here
    const bool few = CL == 1 && total <= WARPS;
    if (me == 0 && threadIdx.x == 0) {
        a.count[list_no] = few ? 0 : total;
        if (h == 0) a.info[b] = make_int4(c.budget, c.settled, c.base, 0);
    }
    // positions of slots that had none, once nobody reads any
    if (CL > 1) cluster.sync();
    if (a.positions.p)
        for (int s = max(c.settled, f0) + (int)threadIdx.x; s < min(c.budget, f1); s += THREADS) {
            const int index = page_index(a.pages, s), page = named(a.pages, table_entry(a.seq, b, index));
            if (page >= 0) reinterpret_cast<int32_t*>(a.positions.p)[slot_offset(a.positions, page, s - index * a.pages.page_size, h)] = c.base + s;
        }
    if (few) {
        __syncthreads();
        if (warp < total) move_one<VEC>(a, elem, b, h, c, list[warp], lane);
    }
}

// A warp takes up to 32 moves of a list at a time: each lane looks up one of them and moves its score and position, then all lanes move the rows together, four loads of each under way.
constexpr int MOVE_THREADS = 256, MOVE_AHEAD = 4;
template <int VEC>
__global__ void __launch_bounds__(MOVE_THREADS, 5) k_evict_move(const __grid_constant__ EvictArgs a, int elem, int blocks, int row_shift) {
    typedef typename Unit<VEC>::T U;
    const int list = blockIdx.x / blocks, part = blockIdx.x - list * blocks;
    const int b = list / a.Hkv, h = list - b * a.Hkv, lane = threadIdx.x & 31;
    pdl_wait();
    const int n = min(a.count[list], a.list_cap);
    const bool tells = part == 0 && h == 0 && threadIdx.x == 0;
    if (n == 0 && !tells) return;
    const int4 info = a.info[b];
    if (tells) {
        a.kv_out[b] = info.x < 0 ? a.seq.kv_len[b] : info.x;
        if (a.settled && info.x >= 0) a.settled[b] = info.x;
    }
    const int warps = blocks * (MOVE_THREADS / 32), each = min(32, (n + warps - 1) / warps);
    const int2* moves = a.list + (size_t)list * a.list_cap;
    for (long long m0 = (long long)(part * (MOVE_THREADS / 32) + (int)(threadIdx.x >> 5)) * each; m0 < n; m0 += (long long)warps * each) {
        const int have = (int)min((long long)each, n - m0);
        long long from = 0, to = -1;                // bytes behind k and behind v
        if (lane < have) {
            int2 x = moves[m0 + lane];
            x.x = min(max(x.x, 0), a.seq.kv_cap - 1);
            x.y = min(max(x.y, 0), a.seq.kv_cap - 1);
            const int fi = page_index(a.pages, x.x), ti = page_index(a.pages, x.y), fs = x.x - fi * a.pages.page_size, ts = x.y - ti * a.pages.page_size;
            int fp = table_entry(a.seq, b, fi), tp = table_entry(a.seq, b, ti);
            fp = named(a.pages, fp);
            tp = named(a.pages, tp);
            if (fp < 0 || tp < 0) set_error(a.seq.status, DEV_E_INDEX);
            else {
                from = (long long)row_offset(a.pages, fp, fs, h) * elem;
                to = (long long)row_offset(a.pages, tp, ts, h) * elem;
                const float score = reinterpret_cast<const float*>(a.scores.p)[slot_offset(a.scores, fp, fs, h)];
                int pos = info.z + x.x;
                if (a.positions.p && x.x < info.y) pos = reinterpret_cast<const int32_t*>(a.positions.p)[slot_offset(a.positions, fp, fs, h)];
                reinterpret_cast<float*>(a.scores.p)[slot_offset(a.scores, tp, ts, h)] = score;
                if (a.positions.p) reinterpret_cast<int32_t*>(a.positions.p)[slot_offset(a.positions, tp, ts, h)] = pos;
            }
        }
        const int units = 2 << row_shift, items = have * units;     // units of keys, then of values, move after move
        for (int i0 = 0; i0 < items; i0 += 32 * MOVE_AHEAD) {
            U v[MOVE_AHEAD];
            char* dst[MOVE_AHEAD];
#pragma unroll
            for (int j = 0; j < MOVE_AHEAD; ++j) {
                const int i = i0 + j * 32 + lane, mv = (i >> (row_shift + 1)) & 31, u = i & (units - 1);
                const long long f = __shfl_sync(0xffffffffu, from, mv), t = __shfl_sync(0xffffffffu, to, mv);
                char* base = reinterpret_cast<char*>(u >> row_shift ? a.pages.v : a.pages.k) + (size_t)(u & ((1 << row_shift) - 1)) * VEC;
                dst[j] = i < items && t >= 0 ? base + t : nullptr;
                if (dst[j]) v[j] = *reinterpret_cast<const U*>(base + f);
            }
#pragma unroll
            for (int j = 0; j < MOVE_AHEAD; ++j)
                if (dst[j]) *reinterpret_cast<U*>(dst[j]) = v[j];
        }
    }
}

// ---- acceptance: a block per sequence; its first warp walks the tree, four rows a lane
constexpr int ACCEPT_THREADS = 256;
template <int VEC>
__global__ void __launch_bounds__(ACCEPT_THREADS) k_paged_accept(const __grid_constant__ AcceptArgs a, int elem) {
    typedef typename Unit<VEC>::T U;
    __shared__ int s_chosen[RT], s_path[RT], s_n, s_top;
    const int b = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // whether an earlier sequence reaches into this one: as load_seq has it
    int top = 0;
    for (int i = threadIdx.x; i < b; i += ACCEPT_THREADS) {
        const int start = __ldg(a.seq.q_start + i), end = __ldg(a.seq.q_start + i + 1), kv = __ldg(a.seq.kv_len + i);
        if (start >= 0 && end >= start && end <= a.seq.n_tokens && end - start <= a.seq.max_new && kv >= 0 && kv <= a.seq.kv_cap) top = max(top, end);
    }
    if (threadIdx.x == 0) s_top = 0;
    __syncthreads();
    top = (int)__reduce_max_sync(0xffffffffu, (unsigned)top);
    if (lane == 0 && top) atomicMax(&s_top, top);
    __syncthreads();
    top = s_top;
    bool odd;
    Seq s = load_seq(a.seq, b, top, odd);
    if (s.n > s.kv) {
        set_error(a.seq.status, DEV_E_INDEX);
        s.n = 0;
    }
    for (int i = threadIdx.x; i < s.n; i += ACCEPT_THREADS) s_chosen[i] = __ldg(a.chosen + s.start + i);
    __syncthreads();
    if (warp == 0) {
        int parent[4], token[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = j * 32 + lane;
            parent[j] = -1;
            token[j] = -1;
            if (i > 0 && i < s.n) {
                parent[j] = __ldg(a.parents + s.start + i);
                token[j] = __ldg(a.drafted + s.start + i);
                if (parent[j] >= i) parent[j] = -1;         // (rows only hang on earlier ones: the walk goes forward)
            }
        }
        int n = 0;
        for (int at = s.n > 0 ? 0 : -1; at >= 0;) {
            const int want = s_chosen[at];
            if (lane == 0) s_path[n] = at;
            ++n;
            int next = -1;
            if (want >= 0) {
#pragma unroll
                for (int j = 3; j >= 0; --j) {
                    const uint32_t fits = __ballot_sync(0xffffffffu, parent[j] == at && token[j] == want);
                    if (fits) next = j * 32 + __ffs(fits) - 1;
                }
            }
            at = next;
        }
        if (lane == 0) s_n = n;
    }
    __syncthreads();
    const int n = s_n, L = s.kv - s.n;
    for (int i = threadIdx.x; i < a.out_stride; i += ACCEPT_THREADS) {
        const int row = i < n ? s_path[i] : -1, token = row >= 0 ? s_chosen[row] : -1;
        a.tokens_out[(size_t)b * a.out_stride + i] = token < 0 ? -1 : token;
        if (a.rows_out) a.rows_out[(size_t)b * a.out_stride + i] = row;
    }
    if (threadIdx.x == 0) {
        a.n_out[b] = n > 0 && s_chosen[s_path[n - 1]] < 0 ? n - 1 : n;
        a.kv_out[b] = s.n > 0 ? L + n : __ldg(a.seq.kv_len + b);
    }
    // rows of the path to their positions, one after the other: a row comes from behind the place of every later one.  Each thread keeps to
    // its own units, so nobody waits
    const int row = a.D * elem / VEC, units = a.Hkv * 2 * row;
    for (int u = threadIdx.x; u < units; u += ACCEPT_THREADS) {
        const int h = u / (2 * row), r = u - h * 2 * row;
        char* base = reinterpret_cast<char*>(r < row ? a.pages.k : a.pages.v) + (size_t)(r < row ? r : r - row) * VEC;
        for (int i = 1; i < n; ++i) {
            const int from = L + s_path[i], to = L + i;
            if (from == to) continue;
            const int fi = page_index(a.pages, from), ti = page_index(a.pages, to);
            const int fp = load_page(a.seq, a.pages, b, fi), tp = load_page(a.seq, a.pages, b, ti);
            if (fp < 0 || tp < 0) continue;
            *reinterpret_cast<U*>(base + row_offset(a.pages, tp, to - ti * a.pages.page_size, h) * elem) =
                *reinterpret_cast<const U*>(base + row_offset(a.pages, fp, from - fi * a.pages.page_size, h) * elem);
        }
    }
}


template <int VEC>
cudaError_t run_select(const EvictArgs& a, int elem, int cl, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.seq.batch * a.Hkv) * cl);
    cfg.blockDim = dim3(SELECT_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cl;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_evict_select<VEC>, a, elem);
}
template <int VEC>
int run_evict(EvictArgs a, int elem, int n_sm, cudaStream_t s) {
    const int lists = a.seq.batch * a.Hkv, cl = evict_blocks(a.seq.kv_cap, a.list_cap, lists, n_sm, &a.as_needed);
    if (run_select<VEC>(a, elem, cl, s) != cudaSuccess) return -1;
    const long long want = (long long)n_sm * 8 / lists;
    const int blocks = want < 1 ? 1 : (int)want;
    return launch_k(k_evict_move<VEC>, dim3((unsigned)lists * blocks), dim3(MOVE_THREADS), 0, s, true, a, elem, blocks, shift_of(a.D * elem / VEC)) != cudaSuccess;
}

}  // namespace

int launch_evict(int dtype, const EvictArgs& a, int n_sm, cudaStream_t s) {
    const int elem = dtype == 0 ? 4 : 2;
    switch (a.vec * elem) {
        case 16: return run_evict<16>(a, elem, n_sm, s);
        case 8: return run_evict<8>(a, elem, n_sm, s);
        case 4: return run_evict<4>(a, elem, n_sm, s);
        default: return run_evict<2>(a, elem, n_sm, s);
    }
}

int launch_accept(int dtype, const AcceptArgs& a, cudaStream_t s) {
    const int elem = dtype == 0 ? 4 : 2;
    switch (a.vec * elem) {
        case 16: k_paged_accept<16><<<a.seq.batch, ACCEPT_THREADS, 0, s>>>(a, elem); break;
        case 8: k_paged_accept<8><<<a.seq.batch, ACCEPT_THREADS, 0, s>>>(a, elem); break;
        case 4: k_paged_accept<4><<<a.seq.batch, ACCEPT_THREADS, 0, s>>>(a, elem); break;
        default: k_paged_accept<2><<<a.seq.batch, ACCEPT_THREADS, 0, s>>>(a, elem);
    }
    return 0;
}

}  // namespace esp
