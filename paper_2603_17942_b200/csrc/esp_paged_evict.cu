// Cutting caches to their budgets, and the acceptance of draft trees: the two operators that move slots of a paged cache.
//
// Eviction: a list of a sequence and KV head is a choice of its `budget` largest keys (score, recency), 32-bit numbers in the order of
// the scores.  k_evict_select finds the smallest key that stays by its digits, 11 + 11 + 10 bits, with histograms in shared memory, then deals the
// kept slots behind the budget to the dropped ones in front of it, both in order, so the answer depends on nothing but the numbers.
// k_evict_move moves the rows of all lists, spread over the whole GPU.
#include "esp_paged.cuh"

namespace esp {

namespace {

using namespace paged;

__device__ __forceinline__ size_t slot_offset(const SlotsView& v, int page, int slot, int head) {
    return (size_t)((long long)page * v.page + (long long)slot * v.tok + (long long)head * v.head);
}
__device__ __forceinline__ size_t row_offset(const PagesView& v, int page, int slot, int head) {
    return (size_t)((long long)page * v.page + (long long)slot * v.tok + (long long)head * v.head);
}

// Larger numbers for larger scores, equal ones for equal scores (-0 = 0); a NaN as -infinity.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) x = -INFINITY;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t KEY_INF = 0xff800000u;      // order_key(INFINITY)

constexpr int SELECT_THREADS = 1024, SELECT_WARPS = SELECT_THREADS / 32;
constexpr int KEYS_IN_SMEM = 48 * 1024;        // keys of longer lists are made anew in every pass
constexpr int BINS = 2048;

struct SeqCut {
    int kv, budget, seen, settled;
    bool cut;
};
__device__ __forceinline__ SeqCut load_cut(const EvictArgs& a, int b) {
    SeqCut c;
    c.kv = __ldg(a.seq.kv_len + b);
    c.budget = __ldg(a.budget + b);
    c.seen = a.positions.p ? __ldg(a.seen + b) : c.kv;
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
__device__ __forceinline__ int position_of(const EvictArgs& a, const SeqCut& c, int s, int page, int slot, int head) {
    if (a.positions.p && s < c.settled) return page < 0 ? -1 : reinterpret_cast<const int32_t*>(a.positions.p)[slot_offset(a.positions, page, slot, head)];
    return c.seen - c.kv + s;
}

__global__ void __launch_bounds__(SELECT_THREADS) k_evict_select(const __grid_constant__ EvictArgs a) {
    extern __shared__ uint32_t s_key[];                 // [min(kv, KEYS_IN_SMEM)]
    __shared__ uint32_t s_hist[BINS];
    __shared__ int s_warp[SELECT_WARPS + 1], s_warp2[SELECT_WARPS + 1];
    __shared__ int s_bin, s_above;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = blockIdx.x / a.Hkv, h = blockIdx.x - b * a.Hkv;
    pdl_launch_dependents();
    const SeqCut c = load_cut(a, b);
    if (!c.cut) {
        if (threadIdx.x == 0) {
            a.count[blockIdx.x] = 0;
            if (h == 0) a.len[b] = -1;
        }
        return;
    }
    const bool kept_in_smem = c.kv <= KEYS_IN_SMEM;
    auto make_key = [&](int s) {
        const int index = page_index(a.pages, s), slot = s - index * a.pages.page_size;
        const int page = load_page(a.seq, a.pages, b, index);
        const float x = page < 0 ? -INFINITY : reinterpret_cast<const float*>(a.scores.p)[slot_offset(a.scores, page, slot, h)];
        // (positions differ, so they are told apart in 64 bits)
        if ((long long)position_of(a, c, s, page, slot, h) >= (long long)c.seen - a.recent) return KEY_INF;
        return order_key(x);
    };
    auto key = [&](int s) { return kept_in_smem ? s_key[s] : make_key(s); };
    if (kept_in_smem)
        for (int s = threadIdx.x; s < c.kv; s += SELECT_THREADS) s_key[s] = make_key(s);

    // ---- the smallest key that stays, `top`, and how many keys are above it
    uint32_t top = 0, mask = 0;
    int above = 0;
    constexpr int SHIFT[3] = {21, 10, 0}, WIDTH[3] = {11, 11, 10};
#pragma unroll 1
    for (int d = 0; d < 3; ++d) {
        for (int i = threadIdx.x; i < BINS; i += SELECT_THREADS) s_hist[i] = 0;
        __syncthreads();
        const uint32_t digit = (1u << WIDTH[d]) - 1u;
        for (int s = threadIdx.x; s < c.kv; s += SELECT_THREADS) {
            const uint32_t k = key(s);
            if ((k & mask) == top) atomicAdd(&s_hist[(k >> SHIFT[d]) & digit], 1u);
        }
        __syncthreads();
        // bins from the top: thread t has bins BINS - 1 - 2t and the one below
        const int hi = BINS - 1 - 2 * threadIdx.x;
        const int n0 = (int)s_hist[hi], n1 = (int)s_hist[hi - 1];
        const int incl = (int)warp_scan_u32(n0 + n1, lane);
        if (lane == 31) s_warp[warp] = incl;
        __syncthreads();
        if (warp == 0) {
            const int x = s_warp[lane], y = (int)warp_scan_u32(x, lane);
            s_warp[lane] = y - x;
        }
        __syncthreads();
        const int before = above + s_warp[warp] + incl - n0 - n1;
        if (before < c.budget && c.budget <= before + n0) { s_bin = hi; s_above = before; }
        else if (before + n0 < c.budget && c.budget <= before + n0 + n1) { s_bin = hi - 1; s_above = before + n0; }
        if (c.budget == 0 && threadIdx.x == 0) { s_bin = BINS - 1; s_above = 0; }
        __syncthreads();
        above = s_above;
        top |= ((uint32_t)s_bin & digit) << SHIFT[d];
        mask |= digit << SHIFT[d];
    }
    const int ties = c.budget - above;                  // slots with the key `top` that stay: the first ones

    // ---- each warp has a stretch of slots: ties in front of it, then kept ones behind the budget and dropped ones before it
    const int each = (c.kv + SELECT_THREADS - 1) / SELECT_THREADS * 32, s0 = min(c.kv, warp * each), s1 = min(c.kv, s0 + each);
    auto block_before = [&](int* of, int mine) {        // the sum over the warps in front (mine: the same in every lane)
        if (lane == 0) of[warp] = mine;
        __syncthreads();
        int before = 0;
        for (int w = 0; w < warp; ++w) before += of[w];
        return before;
    };
    int n = 0;
    for (int i = s0; i < s1; i += 32) n += __popc(__ballot_sync(0xffffffffu, i + lane < s1 && key(min(i + lane, s1 - 1)) == top));
    const int tie0 = block_before(s_warp, n);
    __syncthreads();
    int moves = 0, holes = 0, tie = tie0;
    auto kept = [&](int s, uint32_t k, bool in) {       // all lanes
        const uint32_t same = __ballot_sync(0xffffffffu, in && k == top);
        const bool stays = in && (k > top || (k == top && tie + __popc(same & ((1u << lane) - 1u)) < ties));
        tie += __popc(same);
        return stays;
    };
    for (int i = s0; i < s1; i += 32) {
        const int s = i + lane;
        const bool in = s < s1, stays = kept(s, in ? key(s) : 0u, in);
        moves += __popc(__ballot_sync(0xffffffffu, stays && s >= c.budget));
        holes += __popc(__ballot_sync(0xffffffffu, in && !stays && s < c.budget));
    }
    int m = block_before(s_warp, moves), e = block_before(s_warp2, holes);
    int2* list = a.list + (size_t)blockIdx.x * a.list_cap;
    tie = tie0;
    for (int i = s0; i < s1; i += 32) {
        const int s = i + lane;
        const bool in = s < s1, stays = kept(s, in ? key(s) : 0u, in);
        const uint32_t go = __ballot_sync(0xffffffffu, stays && s >= c.budget), to = __ballot_sync(0xffffffffu, in && !stays && s < c.budget);
        const uint32_t low = (1u << lane) - 1u;
        if ((go >> lane) & 1) list[m + __popc(go & low)].x = s;
        if ((to >> lane) & 1) list[e + __popc(to & low)].y = s;
        m += __popc(go);
        e += __popc(to);
    }
    if (threadIdx.x == SELECT_THREADS - 1) {            // (the last warp has them all in front of it)
        a.count[blockIdx.x] = m;
        if (h == 0) a.len[b] = c.budget;
        s_bin = m;
    }
    __syncthreads();
    // ---- scores and positions
    const int total = s_bin;
    if (a.positions.p)
        for (int s = max(c.settled, 0) + (int)threadIdx.x; s < c.budget; s += SELECT_THREADS) {
            const int index = page_index(a.pages, s), page = load_page(a.seq, a.pages, b, index);
            if (page >= 0) reinterpret_cast<int32_t*>(a.positions.p)[slot_offset(a.positions, page, s - index * a.pages.page_size, h)] = c.seen - c.kv + s;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < total; i += SELECT_THREADS) {
        const int2 x = list[i];
        const int fi = page_index(a.pages, x.x), ti = page_index(a.pages, x.y), fs = x.x - fi * a.pages.page_size, ts = x.y - ti * a.pages.page_size;
        const int fp = load_page(a.seq, a.pages, b, fi), tp = load_page(a.seq, a.pages, b, ti);
        if (tp < 0) continue;
        reinterpret_cast<float*>(a.scores.p)[slot_offset(a.scores, tp, ts, h)] =
            fp < 0 ? -INFINITY : reinterpret_cast<const float*>(a.scores.p)[slot_offset(a.scores, fp, fs, h)];
        if (a.positions.p) reinterpret_cast<int32_t*>(a.positions.p)[slot_offset(a.positions, tp, ts, h)] = position_of(a, c, x.x, fp, fs, h);
    }
}

// Row of `bytes` bytes, VEC of them to a lane; lanes of a group that covers the row
template <int VEC> struct Unit;
template <> struct Unit<16> { typedef uint4 T; };
template <> struct Unit<8> { typedef uint2 T; };
template <> struct Unit<4> { typedef uint32_t T; };
template <> struct Unit<2> { typedef uint16_t T; };

constexpr int MOVE_THREADS = 256;
template <int VEC>
__global__ void __launch_bounds__(MOVE_THREADS) k_evict_move(const __grid_constant__ EvictArgs a, int elem, int blocks) {
    typedef typename Unit<VEC>::T U;
    const int list = blockIdx.x / blocks, part = blockIdx.x - list * blocks;
    const int b = list / a.Hkv, h = list - b * a.Hkv;
    pdl_wait();
    if (part == 0 && h == 0 && threadIdx.x == 0) {
        const int len = a.len[b];
        a.kv_out[b] = len < 0 ? a.seq.kv_len[b] : len;
        if (a.settled && len >= 0) a.settled[b] = len;
    }
    const int n = a.count[list], row = a.D * elem / VEC;            // units of a row
    const int2* moves = a.list + (size_t)list * a.list_cap;
    const long long items = (long long)n * row * 2;                 // units of keys, then of values, move after move
    for (long long i = (long long)part * MOVE_THREADS + threadIdx.x; i < items; i += (long long)blocks * MOVE_THREADS) {
        const int mv = (int)(i / (2 * row)), r = (int)(i - (long long)mv * 2 * row);
        const int2 x = moves[mv];
        const int fi = page_index(a.pages, x.x), ti = page_index(a.pages, x.y);
        const int fp = load_page(a.seq, a.pages, b, fi), tp = load_page(a.seq, a.pages, b, ti);
        if (fp < 0 || tp < 0) continue;
        char* base = reinterpret_cast<char*>(r < row ? a.pages.k : a.pages.v);
        const int u = r < row ? r : r - row;
        const U v = *reinterpret_cast<const U*>(base + row_offset(a.pages, fp, x.x - fi * a.pages.page_size, h) * elem + (size_t)u * VEC);
        *reinterpret_cast<U*>(base + row_offset(a.pages, tp, x.y - ti * a.pages.page_size, h) * elem + (size_t)u * VEC) = v;
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

}  // namespace

int launch_evict(int dtype, const EvictArgs& a, int n_sm, cudaStream_t s) {
    const int lists = a.seq.batch * a.Hkv, elem = dtype == 0 ? 4 : 2;
    const int keys = a.seq.kv_cap < KEYS_IN_SMEM ? a.seq.kv_cap : KEYS_IN_SMEM;
    if (ensure_dynamic_smem(reinterpret_cast<const void*>(&k_evict_select), KEYS_IN_SMEM * 4)) return -1;
    k_evict_select<<<lists, SELECT_THREADS, keys * 4, s>>>(a);
    const long long want = (long long)n_sm * 8 / lists;
    const int blocks = want < 1 ? 1 : (int)want;
    const dim3 grid((unsigned)lists * blocks), block(MOVE_THREADS);
    cudaError_t e;
    switch (a.vec * elem) {
        case 16: e = launch_k(k_evict_move<16>, grid, block, 0, s, true, a, elem, blocks); break;
        case 8: e = launch_k(k_evict_move<8>, grid, block, 0, s, true, a, elem, blocks); break;
        case 4: e = launch_k(k_evict_move<4>, grid, block, 0, s, true, a, elem, blocks); break;
        default: e = launch_k(k_evict_move<2>, grid, block, 0, s, true, a, elem, blocks);
    }
    return e != cudaSuccess;
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
