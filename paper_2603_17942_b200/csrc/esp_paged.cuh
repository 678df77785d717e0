// How the attention over pages deals its work, shared by its kernels.
//
// The pairs (token, query head) of one sequence and KV head are cut into tiles of `rows` tokens; a tile has to walk the chunks of CK
// keys that any of its tokens can see.  All (sequence, KV head, tile, chunk) units of the batch form one line, and CTA c takes the units
// [W c / G, W (c + 1) / G): every CTA gets the same number of chunks whatever the lengths are, and nobody on the host has to know
// them.  A tile that lies in one CTA is finished there; the pieces of a tile that several CTAs share are stored as split partials
// (weighted values, maximum, sum) and joined by the merge kernel in the order of the CTAs, so a call always gives the same bits.
// A CTA's pieces of shared tiles are its first and its last, so two slots per CTA are enough.
#pragma once

#include "esp_paged.h"

namespace esp {
namespace paged {

constexpr int KV_LIMIT = 1 << 30;

// A sequence as the device reads it, checked; a description that does not hold together leaves the sequence without tokens.
struct Seq {
    int start, n, kv;     // first token, tokens, cached positions with them
};
__device__ __forceinline__ Seq load_seq(const SeqTable& t, int b) {
    Seq s;
    s.start = __ldg(t.q_start + b);
    const int end = __ldg(t.q_start + b + 1);
    s.kv = __ldg(t.kv_len + b);
    const bool ok = s.start >= 0 && end >= s.start && end <= t.n_tokens && end - s.start <= t.max_new && s.kv >= 0 && s.kv <= t.kv_cap;
    s.n = ok ? end - s.start : 0;
    if (!ok) set_error(t.status, DEV_E_INDEX);
    return s;
}
// the page of a position < kv_len, -1 if the table names none
__device__ __forceinline__ int load_page(const SeqTable& t, const PagesView& p, int b, int index) {
    const int page = __ldg(t.table + (size_t)b * t.table_stride + index);
    if (page >= 0 && page < p.n_pages) return page;
    set_error(t.status, DEV_E_INDEX);
    return -1;
}

struct Tile {
    int r0, nr, c0, nc;   // tokens [r0, r0 + nr), chunks [c0, c0 + nc), nc >= 1 (a tile that sees nothing has one chunk without visible keys)
};
template <int CK>
__device__ __forceinline__ Tile make_tile(const PagedAttnArgs& a, const Seq& s, int t) {
    Tile x;
    x.r0 = t * a.rows;
    x.nr = min(a.rows, s.n - x.r0);
    const int L = s.kv - s.n;
    const int hi = max(0, a.anc ? s.kv : L + x.r0 + x.nr);
    const int lo = a.window > 0 ? max(0, L + x.r0 - a.window + 1) : 0;
    x.c0 = lo / CK;
    x.nc = max(1, (hi + CK - 1) / CK - x.c0);
    return x;
}
__device__ __forceinline__ int n_tiles(const PagedAttnArgs& a, const Seq& s) { return (s.n + a.rows - 1) / a.rows; }

// Where a unit lies: everything a CTA needs to walk on from there.
struct Cursor {
    long long tile_u;     // first unit of the tile
    int b, kvh, t;
    Seq s;
    Tile x;
};
struct Deal {             // in shared memory, filled by deal()
    long long total;
    int ctas;             // CTAs that take part: each of them has at least one unit
    Cursor at;            // the tile that holds the unit asked for
    long long scan[32];
    long long unit;
    int owner, owner_b;
    long long owner_rest, owner_u;
};

__device__ __forceinline__ long long cta_begin(long long total, int ctas, int c) { return total * c / ctas; }
__device__ __forceinline__ int cta_of_unit(long long total, int ctas, long long u) { return (int)(((u + 1) * ctas + total - 1) / total - 1); }

// Chunks of all tiles of a sequence (one KV head).  All 32 lanes call it together with a sequence each; long ones are counted by the whole warp.
template <int CK>
__device__ __forceinline__ long long seq_chunks(const PagedAttnArgs& a, const Seq& s, int lane) {
    const int T = n_tiles(a, s);
    long long w = 0;
    if (T <= 16)
        for (int t = 0; t < T; ++t) w += make_tile<CK>(a, s, t).nc;
    for (uint32_t big = __ballot_sync(0xffffffffu, T > 16); big; big &= big - 1) {
        const int src = __ffs(big) - 1;
        Seq o;
        o.start = 0;
        o.n = __shfl_sync(0xffffffffu, s.n, src);
        o.kv = __shfl_sync(0xffffffffu, s.kv, src);
        const int To = n_tiles(a, o);
        long long p = 0;
        for (int t = lane; t < To; t += 32) p += make_tile<CK>(a, o, t).nc;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) p += __shfl_xor_sync(0xffffffffu, p, d);
        if (lane == src) w = p;
    }
    return w;
}

// Called by all threads of a block (a multiple of 32, at most 1024): counts the batch's units and finds the tile that holds the first unit of
// CTA `cta` (or, LAST, the last unit of it).  false: the CTA has no units.
template <int CK, bool LAST>
__device__ __forceinline__ bool deal(const PagedAttnArgs& a, int cta, int min_units, Deal* d) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    const int per = (a.seq.batch + blockDim.x - 1) / blockDim.x;        // consecutive sequences of a thread
    const int b0 = min((int)threadIdx.x * per, a.seq.batch), b1 = min(b0 + per, a.seq.batch);
    long long mine = 0;
    for (int i = 0; i < per; ++i) {                                      // the same trips in every lane
        Seq s;
        s.start = s.n = s.kv = 0;
        if (b0 + i < b1) s = load_seq(a.seq, b0 + i);
        mine += seq_chunks<CK>(a, s, lane) * a.Hkv;
    }
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) d->scan[warp] = incl;
    __syncthreads();
    long long before = incl - mine, total = 0;
    for (int w = 0; w < n_warps; ++w) {
        if (w < warp) before += d->scan[w];
        total += d->scan[w];
    }
    const int ctas = (int)max(1ll, min((long long)a.n_cta, (total + min_units - 1) / min_units));
    if (total == 0 || cta >= ctas) return false;                         // the same answer in every thread
    const long long unit = LAST ? cta_begin(total, ctas, cta + 1) - 1 : cta_begin(total, ctas, cta);
    if (before <= unit && unit < before + mine) {
        d->total = total;
        d->ctas = ctas;
        d->unit = unit;
        d->owner = threadIdx.x;
        d->owner_b = b0;
        d->owner_u = before;
    }
    __syncthreads();
    if (warp == (d->owner >> 5)) {
        // the warp walks the owner's sequences, then the tiles of the one that holds the unit
        long long u0 = d->owner_u;
        int b = d->owner_b;
        Seq s;
        long long Wt;
        for (;; ++b) {
            s = load_seq(a.seq, b);                                      // the same sequence in every lane
            Wt = 0;
            const int T = n_tiles(a, s);
            for (int t = lane; t < T; t += 32) Wt += make_tile<CK>(a, s, t).nc;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) Wt += __shfl_xor_sync(0xffffffffu, Wt, o);
            if (unit < u0 + Wt * a.Hkv) break;
            u0 += Wt * a.Hkv;
        }
        const int kvh = (int)((unit - u0) / Wt);
        u0 += kvh * Wt;
        for (int t0 = 0;; t0 += 32) {
            const int t = t0 + lane;
            int nc = 0;
            if (t < n_tiles(a, s)) nc = make_tile<CK>(a, s, t).nc;
            long long in = nc;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(0xffffffffu, in, o);
                if (lane >= o) in += v;
            }
            const bool here = unit >= u0 + in - nc && unit < u0 + in;
            if (here) {
                d->at.tile_u = u0 + in - nc;
                d->at.b = b;
                d->at.kvh = kvh;
                d->at.t = t;
                d->at.s = s;
                d->at.x = make_tile<CK>(a, s, t);
            }
            if (__ballot_sync(0xffffffffu, here)) break;
            u0 += __shfl_sync(0xffffffffu, in, 31);
        }
    }
    __syncthreads();
    return true;
}

template <int CK>
__device__ __forceinline__ void next_tile(const PagedAttnArgs& a, Cursor& c) {
    c.tile_u += c.x.nc;
    if (++c.t >= n_tiles(a, c.s)) {
        c.t = 0;
        if (++c.kvh >= a.Hkv) {
            c.kvh = 0;
            do {
                if (++c.b >= a.seq.batch) return;                        // the end of the line: nobody looks at the tile
                c.s = load_seq(a.seq, c.b);
            } while (c.s.n == 0);
        }
    }
    c.x = make_tile<CK>(a, c.s, c.t);
}

// One piece of a CTA: chunks [c0, c0 + n) of the cursor's tile.
struct Piece {
    int c0, n;
    int slot;             // -1: the whole tile, finished here; else the CTA's slot for the split partial
};
__device__ __forceinline__ Piece make_piece(const Cursor& c, long long begin, long long u, long long end) {
    Piece p;
    const int off = (int)(u - c.tile_u);
    p.n = (int)min((long long)(c.x.nc - off), end - u);
    p.c0 = c.x.c0 + off;
    p.slot = p.n == c.x.nc ? -1 : (begin >= c.tile_u ? 0 : 1);
    return p;
}

// What token i of its sequence sees of position pos (< kv).
struct RowMask {
    int lo, hi;                        // positions [lo, hi) without a tree; with one [0, L) and the bits
    unsigned long long b0, b1;
};
__device__ __forceinline__ RowMask row_mask(const PagedAttnArgs& a, const Seq& s, int i) {
    RowMask m;
    const int L = s.kv - s.n, P = L + i;
    m.b0 = m.b1 = 0;
    if (P < 0) {                       // padding sees nothing
        m.lo = m.hi = 0;
    } else if (a.anc) {
        m.lo = 0;
        m.hi = max(L, 0);
        m.b0 = __ldg(a.anc + 2 * (size_t)(s.start + i));
        m.b1 = __ldg(a.anc + 2 * (size_t)(s.start + i) + 1);
    } else {
        m.lo = a.window > 0 ? max(0, P - a.window + 1) : 0;
        m.hi = P + 1;
    }
    return m;
}
// L = kv - n of the sequence
__device__ __forceinline__ bool sees(const RowMask& m, int pos, int L, int kv) {
    if (pos >= m.lo && pos < m.hi) return true;
    const int j = pos - L;
    if (pos >= kv || j < 0 || j >= 128) return false;
    return ((j < 64 ? m.b0 >> j : m.b1 >> (j - 64)) & 1ull) != 0;
}

// where pair p of the tile's (token, head) pairs goes
__device__ __forceinline__ size_t out_offset(const HeadsView& v, int token, int head) { return (size_t)((long long)token * v.tok + (long long)head * v.head); }

}  // namespace paged
}  // namespace esp
