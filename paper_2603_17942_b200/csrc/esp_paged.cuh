// How the attention over pages deals its work, shared by its kernels.
//
// The pairs (token, query head) of one sequence and KV head are cut into tiles of `rows` tokens; a tile has to walk the chunks of CK
// keys that any of its tokens can see.  All (sequence, KV head, tile, chunk) units of the batch form one line, cut into equal shares for
// the CTAs: every CTA gets the same number of chunks, or one more, whatever the lengths are, and nobody on the host has to know them.  A tile that lies in one CTA is finished there; the pieces of a tile that several CTAs share are stored as split partials
// (weighted values, maximum, sum) and joined by the merge kernel in the order of the CTAs, so a call always gives the same bits.
// A CTA's pieces of shared tiles are its first and its last, so two slots per CTA are enough.
#pragma once

#include "esp_paged.h"

namespace esp {
namespace paged {

constexpr int KV_LIMIT = 1 << 30;

// A sequence as the device reads it, checked; a description that does not hold together leaves the sequence without tokens.
// top: the furthest end of the sequences before b that hold together by themselves; b must not start in front of it, or two sequences would own a token.  That can only be
// where some sequence did not hold together, which `odd` tells: callers that start at another sequence than the first pass 0 for top as long as there is none.
struct Seq {
    int start, n, kv;     // first token, tokens, cached positions with them
};
__device__ __forceinline__ Seq load_seq(const SeqTable& t, int b, int& top, bool& odd) {
    Seq s;
    s.start = __ldg(t.q_start + b);
    const int end = __ldg(t.q_start + b + 1);
    s.kv = __ldg(t.kv_len + b);
    const bool alone = s.start >= 0 && end >= s.start && end <= t.n_tokens && end - s.start <= t.max_new && s.kv >= 0 && s.kv <= t.kv_cap;
    const bool ok = alone && s.start >= top;
    if (alone) top = max(top, end);
    s.n = ok ? end - s.start : 0;
    if (!ok) {
        odd = true;
        set_error(t.status, DEV_E_INDEX);
    }
    return s;
}
// the largest value of the lanes before this one, 0 in the first
__device__ __forceinline__ int warp_max_before(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v = max(v, x);
    }
    v = __shfl_up_sync(0xffffffffu, v, 1);
    return lane ? v : 0;
}
__device__ __forceinline__ int page_index(const PagesView& p, int pos) { return p.page_shift >= 0 ? pos >> p.page_shift : pos / p.page_size; }
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
// What the tile whose first token is r0 sees first (0 or less: everything).  The positions before it in its first chunk are not looked up: a server may have given their pages back.
__device__ __forceinline__ int first_seen(const PagedAttnArgs& a, const Seq& s, int r0) { return a.window > 0 ? s.kv - s.n + r0 - a.window + 1 : 0; }
template <int CK>
__device__ __forceinline__ Tile make_tile(const PagedAttnArgs& a, const Seq& s, int t) {
    Tile x;
    x.r0 = t * a.rows;
    x.nr = min(a.rows, s.n - x.r0);
    const int L = s.kv - s.n;
    const int hi = max(0, a.anc ? s.kv : L + x.r0 + x.nr);
    const int lo = max(0, first_seen(a, s, x.r0));
    x.c0 = lo / CK;
    x.nc = max(1, (hi + CK - 1) / CK - x.c0);
    return x;
}
__device__ __forceinline__ int n_tiles(const PagedAttnArgs& a, const Seq& s) { return a.rows_shift >= 0 ? (s.n + a.rows - 1) >> a.rows_shift : (s.n + a.rows - 1) / a.rows; }

// Where a CTA stands on the line: a tile, and the CTA's own range of units.
struct Cursor {
    uint32_t tile_u;      // first unit of the tile
    int b, kvh, t;
    int top;              // as load_seq has it, behind sequence b
    Seq s;
    Tile x;
};
struct Share {            // CTA c of `ctas` has `each` units, the first `more` CTAs one more
    uint32_t each, more;
    int ctas;
    __device__ __forceinline__ uint32_t begin(int c) const { return (uint32_t)c * each + min((uint32_t)c, more); }
    __device__ __forceinline__ int cta_of(uint32_t u) const {
        const uint32_t wide = more * (each + 1);
        return (int)(u < wide ? u / (each + 1) : more + (u - wide) / each);
    }
};
__device__ __forceinline__ uint32_t warp_sum_u32(uint32_t v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ uint32_t warp_scan_u32(uint32_t v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}

// Chunks of all tiles of a sequence (one KV head), 2^31 if a lane's share of them is 2^26 or more.  All 32 lanes call it together with a sequence each; long ones are counted by the whole warp.
template <int CK>
__device__ __forceinline__ uint32_t seq_chunks(const PagedAttnArgs& a, const Seq& s, int lane) {
    const int T = n_tiles(a, s);
    uint32_t w = 0;
    if (T <= 4)
        for (int t = 0; t < T; ++t) w += make_tile<CK>(a, s, t).nc;
    for (uint32_t big = __ballot_sync(0xffffffffu, T > 4); big; big &= big - 1) {
        const int src = __ffs(big) - 1;
        Seq o;
        o.start = 0;
        o.n = __shfl_sync(0xffffffffu, s.n, src);
        o.kv = __shfl_sync(0xffffffffu, s.kv, src);
        const int To = n_tiles(a, o);
        unsigned long long p = 0;
        for (int t = lane; t < To; t += 32) p += make_tile<CK>(a, o, t).nc;
        const bool most = __any_sync(0xffffffffu, p >> 26);              // (32 lanes below 2^26 each stay below 2^31)
        const uint32_t sum = warp_sum_u32((uint32_t)p);
        if (lane == src) w = most ? 1u << 31 : sum;
    }
    return w;
}

// Called by all lanes of a warp, each warp that needs to know for itself (no barrier, nothing shared): counts the batch's units and finds the tile in
// which CTA `cta` starts.  false: the CTA has no units.  A batch of 2^31 units or more is refused on the device.
template <int CK>
__device__ __forceinline__ bool deal(const PagedAttnArgs& a, int cta, int lane, Share& share, Cursor& at) {
    const int per = (a.seq.batch + 31) >> 5;                             // consecutive sequences of a lane
    const int b0 = lane * per;
    uint32_t mine, chunks = 0;
    unsigned long long wide;
    Seq s;
    int top0 = 0, top;                                                   // in front of the lane's sequences, behind them
    for (bool again = false;; again = true) {
        bool odd = false;
        top = top0;
        mine = 0;
        wide = 0;
        for (int i = 0; i < per; ++i) {                                  // the same trips in every lane
            s.start = s.n = s.kv = 0;
            if (b0 + i < a.seq.batch) s = load_seq(a.seq, b0 + i, top, odd);
            chunks = seq_chunks<CK>(a, s, lane);
            const unsigned long long w = (unsigned long long)chunks * a.Hkv;
            wide += w;
            mine += (uint32_t)w;
        }
        if (again || !__any_sync(0xffffffffu, odd)) break;
        top0 = warp_max_before(top, lane);                               // once more, with what stands in front of each lane's sequences
    }
    if (__any_sync(0xffffffffu, wide >> 26)) {                           // (32 lanes below 2^26 each stay below 2^31)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) wide += __shfl_xor_sync(0xffffffffu, wide, o);
        if (wide >> 31) {
            set_error(a.seq.status, DEV_E_CAPACITY);
            return false;
        }
    }
    const uint32_t incl = warp_scan_u32(mine, lane), total = __shfl_sync(0xffffffffu, incl, 31);
    share.ctas = (int)min((uint32_t)a.n_cta, (total + a.min_units - 1) / a.min_units);
    if (cta >= share.ctas) return false;                                 // (nothing to do at all: no CTAs)
    share.each = total / share.ctas;
    share.more = total - share.each * share.ctas;
    const uint32_t unit = share.begin(cta), before = incl - mine;
    const int owner = __ffs(__ballot_sync(0xffffffffu, before <= unit && unit < incl)) - 1;
    uint32_t u0 = __shfl_sync(0xffffffffu, before, owner), Wt;
    at.b = owner * per;
    if (per == 1) {
        at.s.start = __shfl_sync(0xffffffffu, s.start, owner);
        at.s.n = __shfl_sync(0xffffffffu, s.n, owner);
        at.s.kv = __shfl_sync(0xffffffffu, s.kv, owner);
        at.top = __shfl_sync(0xffffffffu, top, owner);
        Wt = __shfl_sync(0xffffffffu, chunks, owner);
    } else {
        at.top = __shfl_sync(0xffffffffu, top0, owner);
        bool odd;
        for (;; ++at.b) {                                                // the same sequence in every lane
            at.s = load_seq(a.seq, at.b, at.top, odd);
            const int T = n_tiles(a, at.s);
            Wt = 0;
            for (int t = lane; t < T; t += 32) Wt += make_tile<CK>(a, at.s, t).nc;
            Wt = warp_sum_u32(Wt);
            if (unit - u0 < Wt * a.Hkv) break;
            u0 += Wt * a.Hkv;
        }
    }
    at.kvh = (int)((unit - u0) / Wt);
    u0 += at.kvh * Wt;
    for (int t0 = 0;; t0 += 32) {
        const int t = t0 + lane;
        const uint32_t nc = t < n_tiles(a, at.s) ? make_tile<CK>(a, at.s, t).nc : 0;
        const uint32_t in = warp_scan_u32(nc, lane);
        const uint32_t here = __ballot_sync(0xffffffffu, unit - u0 < in);  // the first lane behind the unit has its tile
        if (here) {
            const int src = __ffs(here) - 1;
            at.t = t0 + src;
            at.tile_u = u0 + __shfl_sync(0xffffffffu, in - nc, src);
            break;
        }
        u0 += __shfl_sync(0xffffffffu, in, 31);
    }
    at.x = make_tile<CK>(a, at.s, at.t);
    return true;
}

template <int CK>
__device__ __forceinline__ void next_tile(const PagedAttnArgs& a, Cursor& c) {
    c.tile_u += c.x.nc;
    if (++c.t >= n_tiles(a, c.s)) {
        c.t = 0;
        if (++c.kvh >= a.Hkv) {
            c.kvh = 0;
            bool odd;
            do {
                if (++c.b >= a.seq.batch) return;                        // the end of the line: nobody looks at the tile
                c.s = load_seq(a.seq, c.b, c.top, odd);
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
__device__ __forceinline__ Piece make_piece(const Cursor& c, uint32_t begin, uint32_t u, uint32_t end) {
    Piece p;
    const int off = (int)(u - c.tile_u);
    p.n = (int)min((uint32_t)(c.x.nc - off), end - u);
    p.c0 = c.x.c0 + off;
    p.slot = p.n == c.x.nc ? -1 : (begin >= c.tile_u ? 0 : 1);
    return p;
}

// What the merge kernel has to know of the split tiles that CTA `cta` has pieces of: at most one it has the first piece of (its last piece) and one that
// began before it (its first piece).  two: each CTA has two parts.
struct Descs {
    MergeDesc starts, goes_on;
    __device__ __forceinline__ void clear() { starts.parts = goes_on.parts = 0; }
    __device__ __forceinline__ void note(const PagedAttnArgs& a, const Cursor& c, const Share& share, const Piece& p, bool two = false) {
        if (p.slot < 0) return;
        MergeDesc d;
        d.token = c.s.start + c.x.r0;
        d.pairs = c.x.nr * a.group;
        d.head0 = c.kvh * a.group;
        d.first = share.cta_of(c.tile_u);
        d.parts = (share.cta_of(c.tile_u + c.x.nc - 1) - d.first + 1) * 4 + (two ? 2 : 0) + (share.begin(d.first) >= c.tile_u ? 0 : 1);
        if (p.c0 == c.x.c0) starts = d;
        else goes_on = d;
    }
    __device__ __forceinline__ void store(const PagedAttnArgs& a, int cta) const {
        int4* to = reinterpret_cast<int4*>(a.desc + 2 * cta);
        to[0] = make_int4(starts.token, starts.pairs, starts.head0, starts.parts);
        to[1] = make_int4(starts.first, 0, 0, 0);
        to[2] = make_int4(goes_on.token, goes_on.pairs, goes_on.head0, goes_on.parts);
        to[3] = make_int4(goes_on.first, 0, 0, 0);
    }
};
// split partials: quad dq of a pair's weighted values, in the order in which a warp with a lane per pair writes them
__device__ __forceinline__ size_t part_quad(const PagedAttnArgs& a, int cta, int slot, int dq, int pair) {
    return ((size_t)(cta * 2 + slot) * (a.D / 4) + dq) * a.pairs + pair;
}
__device__ __forceinline__ size_t part_row(const PagedAttnArgs& a, int cta, int slot, int pair) { return (size_t)(cta * 2 + slot) * a.pairs + pair; }

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

template <typename T>
__device__ __forceinline__ void store4(T* y, const float4& x, bool vec) {
    if constexpr (sizeof(T) == 4) {
        if (vec) { *reinterpret_cast<float4*>(y) = x; return; }
    } else {
        if (vec) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(x.x, x.y), hi = __floats2bfloat162_rn(x.z, x.w);
            *reinterpret_cast<uint2*>(y) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            return;
        }
    }
    y[0] = from_f32<T>(x.x); y[1] = from_f32<T>(x.y); y[2] = from_f32<T>(x.z); y[3] = from_f32<T>(x.w);
}

}  // namespace paged
}  // namespace esp
