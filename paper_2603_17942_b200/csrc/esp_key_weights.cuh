// How the weights of cached positions are dealt, shared by their kernels.
//
// A position's sum belongs to its key, so here the chunks of CK keys are what is walked: the observed tokens of a sequence are cut into tiles of `rows` tokens, and a chunk
// has to meet the tiles of which some token sees some of its keys; a chunk that none sees has one unit all the same (its numbers are still to be written).  All (sequence, KV
// head, chunk, tile) units of the batch form one line, cut into equal shares for the CTAs.  A chunk that lies in one CTA is finished there; of one that several
// share each CTA stores its sums, and the join adds them in the order of the CTAs: the same call gives the same bits.
#pragma once

#include "esp_paged.cuh"

namespace esp {
namespace paged {

struct WSeq {
    Seq s;
    int i0, T;            // first observed token, tiles of observed tokens
};
struct WChunk {
    int t0, nt;           // tiles [t0, t0 + nt) meet it; nt 0: none does
    __host__ __device__ __forceinline__ int units() const { return max(nt, 1); }
};
// A bound for the observed tokens of a sequence, so that they all are one tile.  (max_new may be far above the tokens of the call; what is added to such a bound has to fit.)
inline int one_tile(const KeyWeightArgs& w) {
    const int most = w.last > 0 && w.last < w.a.seq.max_new ? w.last : w.a.seq.max_new;
    return most < w.a.seq.n_tokens ? most : w.a.seq.n_tokens;
}
// (what does not touch device memory is compiled for the host too, where tests count with it)
__host__ __device__ __forceinline__ WSeq observed(const KeyWeightArgs& w, const Seq& s) {
    WSeq x;
    x.s = s;
    x.i0 = w.last > 0 ? max(0, s.n - w.last) : 0;
    x.T = w.a.rows_shift >= 0 ? (s.n - x.i0 + w.a.rows - 1) >> w.a.rows_shift : (s.n - x.i0 + w.a.rows - 1) / w.a.rows;
    return x;
}
template <int CK>
__host__ __device__ __forceinline__ int n_chunks(const WSeq& x) { return x.T > 0 ? (int)(((unsigned)x.s.kv + CK - 1) / CK) : 0; }
template <int CK>
__host__ __device__ __forceinline__ WChunk make_chunk(const KeyWeightArgs& w, const WSeq& x, int c) {
    WChunk k;
    k.t0 = 0;
    k.nt = x.T;
    if (w.a.anc) return k;
    const long long L = (long long)x.s.kv - x.s.n, p0 = (long long)c * CK, p1 = min(p0 + CK, (long long)x.s.kv);
    const long long first = max(p0 - L, (long long)x.i0);                                                             // the first token that sees the first key
    const long long last = w.a.window > 0 ? min((long long)x.s.n - 1, p1 - 1 + w.a.window - 1 - L) : x.s.n - 1;        // the last one that sees the last key
    if (first > last) k.nt = 0;
    else {
        k.t0 = (int)(first - x.i0) / w.a.rows;
        k.nt = (int)(last - x.i0) / w.a.rows + 1 - k.t0;
    }
    return k;
}
// Units of a sequence (one KV head) whose chunks meet several tiles, counted by a warp; 2^31 if there are as many or more.
template <int CK>
__device__ __forceinline__ uint32_t warp_units(const KeyWeightArgs& w, const WSeq& x, int lane) {
    const int C = n_chunks<CK>(x);
    unsigned long long sum = 0;
    for (int c = lane; c < C; c += 32) sum += make_chunk<CK>(w, x, c).units();
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return sum >> 31 ? 1u << 31 : (uint32_t)sum;
}
// The same for one sequence, by one thread.  A single tile has a unit for each chunk; without a window all chunks up to the first observed token meet all tiles, and where
// only a few chunks are behind that they are counted one by one.  false: there are many to count, n is 0.
template <int CK>
__host__ __device__ __forceinline__ bool lane_units(const KeyWeightArgs& w, const WSeq& x, uint32_t& n) {
    n = 0;
    if (x.T <= 1) {
        n = x.T == 1 ? (uint32_t)n_chunks<CK>(x) : 0u;
        return true;
    }
    const int C = n_chunks<CK>(x);
    // (padding may reach so far that the first tiles see nothing at all: then no chunk meets all of them)
    const int full = w.a.anc ? C : (int)max(0ll, min((long long)C, ((long long)x.s.kv - x.s.n + x.i0 + w.a.rows + CK - 1) / CK));
    if (w.a.window > 0 || C - full > 16) return false;
    unsigned long long sum = (unsigned long long)full * x.T;
    for (int c = full; c < C; ++c) sum += make_chunk<CK>(w, x, c).units();
    n = sum >> 31 ? 1u << 31 : (uint32_t)sum;
    return true;
}
// The same for a sequence of each lane.
template <int CK>
__device__ __forceinline__ uint32_t seq_units(const KeyWeightArgs& w, const WSeq& x, int lane) {
    uint32_t n;
    const bool alone = lane_units<CK>(w, x, n);
    for (uint32_t many = __ballot_sync(0xffffffffu, !alone); many; many &= many - 1) {
        const int src = __ffs(many) - 1;
        WSeq o;
        o.s.start = 0;
        o.s.n = __shfl_sync(0xffffffffu, x.s.n, src);
        o.s.kv = __shfl_sync(0xffffffffu, x.s.kv, src);
        o.i0 = __shfl_sync(0xffffffffu, x.i0, src);
        o.T = __shfl_sync(0xffffffffu, x.T, src);
        const uint32_t sum = warp_units<CK>(w, o, lane);
        if (lane == src) n = sum;
    }
    return n;
}

struct WCursor {
    uint32_t chunk_u;     // first unit of the chunk
    int b, kvh, c;
    int top;
    WSeq x;
    WChunk k;
};

// As deal() of the attention: called by all lanes of a warp; false: the CTA has no units.  2^31 units or more are refused.
template <int CK>
__device__ __forceinline__ bool deal_keys(const KeyWeightArgs& w, int cta, int lane, Share& share, WCursor& at) {
    const PagedAttnArgs& a = w.a;
    const int per = (a.seq.batch + 31) >> 5, b0 = lane * per;
    uint32_t mine = 0, units = 0;
    unsigned long long wide;
    WSeq x;
    int top0 = 0, top;
    for (bool again = false;; again = true) {
        bool odd = false;
        top = top0;
        wide = 0;
        for (int i = 0; i < per; ++i) {
            Seq s;
            s.start = s.n = s.kv = 0;
            if (b0 + i < a.seq.batch) s = load_seq(a.seq, b0 + i, top, odd);
            x = observed(w, s);
            units = seq_units<CK>(w, x, lane);
            wide += (unsigned long long)units * a.Hkv;
            if (wide >> 40) wide = 1ull << 40;               // (enough to be refused)
        }
        if (again || !__any_sync(0xffffffffu, odd)) break;
        top0 = warp_max_before(top, lane);
    }
    mine = (uint32_t)wide;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) wide += __shfl_xor_sync(0xffffffffu, wide, d);
    if (wide >> 31) {
        set_error(a.seq.status, DEV_E_CAPACITY);
        return false;
    }
    const uint32_t incl = warp_scan_u32(mine, lane), total = (uint32_t)wide;
    share.ctas = (int)min((uint32_t)a.n_cta, (total + a.min_units - 1) / a.min_units);
    if (cta >= share.ctas) return false;
    share.each = total / share.ctas;
    share.more = total - share.each * share.ctas;
    const uint32_t unit = share.begin(cta), before = incl - mine;
    const int owner = __ffs(__ballot_sync(0xffffffffu, before <= unit && unit < incl)) - 1;
    uint32_t u0 = __shfl_sync(0xffffffffu, before, owner), U;
    at.b = owner * per;
    if (per == 1) {
        at.x.s.start = __shfl_sync(0xffffffffu, x.s.start, owner);
        at.x.s.n = __shfl_sync(0xffffffffu, x.s.n, owner);
        at.x.s.kv = __shfl_sync(0xffffffffu, x.s.kv, owner);
        at.top = __shfl_sync(0xffffffffu, top, owner);
        U = __shfl_sync(0xffffffffu, units, owner);
        at.x = observed(w, at.x.s);
    } else {
        at.top = __shfl_sync(0xffffffffu, top0, owner);
        bool odd;
        for (;; ++at.b) {                                    // the same sequence in every lane
            at.x = observed(w, load_seq(a.seq, at.b, at.top, odd));
            U = at.x.T == 1 ? (uint32_t)n_chunks<CK>(at.x) : warp_units<CK>(w, at.x, lane);
            if (unit - u0 < U * a.Hkv) break;
            u0 += U * a.Hkv;
        }
    }
    at.kvh = (int)((unit - u0) / U);
    u0 += at.kvh * U;
    if (at.x.T == 1) {
        at.c = (int)(unit - u0);
        at.chunk_u = unit;
    } else {
        for (int c0 = 0;; c0 += 32) {
            const int c = c0 + lane;
            const uint32_t n = c < n_chunks<CK>(at.x) ? make_chunk<CK>(w, at.x, c).units() : 0;
            const uint32_t in = warp_scan_u32(n, lane), here = __ballot_sync(0xffffffffu, unit - u0 < in);
            if (here) {
                const int src = __ffs(here) - 1;
                at.c = c0 + src;
                at.chunk_u = u0 + __shfl_sync(0xffffffffu, in - n, src);
                break;
            }
            u0 += __shfl_sync(0xffffffffu, in, 31);
        }
    }
    at.k = make_chunk<CK>(w, at.x, at.c);
    return true;
}

template <int CK>
__device__ __forceinline__ void next_chunk(const KeyWeightArgs& w, WCursor& k) {
    k.chunk_u += k.k.units();
    if (++k.c >= n_chunks<CK>(k.x)) {
        k.c = 0;
        if (++k.kvh >= w.a.Hkv) {
            k.kvh = 0;
            bool odd;
            do {
                if (++k.b >= w.a.seq.batch) return;
                k.x = observed(w, load_seq(w.a.seq, k.b, k.top, odd));
            } while (n_chunks<CK>(k.x) == 0);
        }
    }
    k.k = make_chunk<CK>(w, k.x, k.c);
}

// The first position that an observed token sees: in front of it a table may name pages that there are no longer, which is no error.
__device__ __forceinline__ int first_observed(const KeyWeightArgs& w, const WSeq& x) { return w.a.window > 0 ? x.s.kv - x.s.n + x.i0 - w.a.window + 1 : 0; }
// The table's entry for position pos (< kv), whatever it says, and where the position's score is; NULL if the entry names no page.
__device__ __forceinline__ int score_entry(const KeyWeightArgs& w, const WCursor& k, int pos) {
    return __ldg(w.a.seq.table + (size_t)k.b * w.a.seq.table_stride + page_index(w.a.pages, pos));
}
__device__ __forceinline__ float* score_of(const KeyWeightArgs& w, const WCursor& k, int pos, int page) {
    if (page < 0 || page >= w.a.pages.n_pages) {
        if (pos >= first_observed(w, k.x)) set_error(w.a.seq.status, DEV_E_INDEX);
        return nullptr;
    }
    return reinterpret_cast<float*>(w.scores.p) + (long long)page * w.scores.page + (long long)(pos - page_index(w.a.pages, pos) * w.a.pages.page_size) * w.scores.tok +
           (long long)k.kvh * w.scores.head;
}
__device__ __forceinline__ float* score_at(const KeyWeightArgs& w, const WCursor& k, int pos) { return score_of(w, k, pos, score_entry(w, k, pos)); }
// whether position pos of the sequence has a score already: new tokens begin at zero
__device__ __forceinline__ bool has_old(const KeyWeightArgs& w, const Seq& s, int pos) { return w.keep != 0.f && pos < s.kv - s.n; }
// What becomes of position pos, given the sum of its weights.
__device__ __forceinline__ void store_score(const KeyWeightArgs& w, const WCursor& k, int pos, float sum) {
    float* y = score_at(w, k, pos);
    if (y) *y = has_old(w, k.x.s, pos) ? fmaf(w.keep, *y, sum) : sum;
}

// One piece of a CTA: tiles [t0, t0 + n) of the cursor's chunk (n 0: the chunk that no tile meets).
struct WPiece {
    int t0, n;
    int slot;             // -1: the whole chunk; else the CTA's slot for its sums
};
__device__ __forceinline__ WPiece make_piece(const WCursor& k, uint32_t begin, uint32_t u, uint32_t end) {
    WPiece p;
    const int off = (int)(u - k.chunk_u), units = (int)min((uint32_t)(k.k.units() - off), end - u);
    p.t0 = k.k.t0 + off;
    p.n = k.k.nt == 0 ? 0 : units;
    p.slot = units == k.k.units() ? -1 : (begin >= k.chunk_u ? 0 : 1);
    return p;
}

}  // namespace paged
}  // namespace esp
