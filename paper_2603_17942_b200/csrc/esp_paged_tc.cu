// Attention over pages on the Blackwell tensor cores: bf16, heads of 64 or 128, blocks of several tokens.
//
// A CTA takes tiles of up to 256 (token, query head) pairs that share a KV head, as two subtiles of 128, and walks their keys 128 at
// a time.  Keys and values come by TMA, page by page (boxes of as many tokens as page size and chunk have in common), into rings of
// stages that both subtiles share:
//   S_s = Q_s K^T    tcgen05.mma, both operands K-major in shared memory, S_s (128 x 128 fp32) in tensor memory;
//   softmax          one thread per pair (= tensor-memory lane): mask, running maximum and sum in the log2 domain, P as bf16 back over S_s;
//   O_s += P_s V     tcgen05.mma with P_s as the tensor-memory operand, V MN-major as the pages have it; O_s stays in tensor memory.
//                    The reference of the exponentials follows the maximum lazily: it moves, and O_s is rescaled, only after a growth of 2^8.
// The tensor cores work on one subtile while the softmax of the other runs; products are issued in the order P_0 V, Q_0 K^T (next chunk),
// P_1 V, Q_1 K^T, and run in that order, so S_s may be overwritten as soon as the P_s V that reads P_s from it has been issued, and S_s
// arriving says that O_s is complete.
// Weights of keys that a pair does not see are zero, but zero times an infinite value is no number: in chunks that not every pair sees
// as a whole, a warp sets values that are no finite numbers to zero in shared memory before the product, and the pairs that see them get them
// when the tile is finished.
// Roles: warps 0 and 2 TMA (keys and queries, values), warp 1 issues the products, warp 3 looks after the values, warps 4-7 and 8-11 softmax and
// output of a subtile.  Every wait is bounded; one that runs out is recorded, the tensor memory is given back and the kernel returns.
//
// What bounds it: 2048 tokens behind 6144, 32/8 heads of 128, take 228 us over the first hundred calls at 1965 MHz, 1.05 PFLOP/s, and 250 to 259 in long rows, where the
// power cap lowers the clock to 1.7 GHz.  A chunk takes a subtile about 3500 cycles: 300 to load the
// scores of a half and find their maximum and 730 for its weights (512 of them the special-function unit's), twice, the last half's product and the next
// scores 770, and the waits between the warps; the tensor cores have 1024 of them for each of the two subtiles, 55 to 60 %.  Built, correct and slower (us
// for the same call): scores of 64 keys in two buffers per subtile, so that the softmax never waits for a product (276: products of 64 keys read the
// queries twice as often, and the issuing warp has twice the hand-overs); a warp of its own for each subtile's products (305: they interleave); a share of
// the exponentials as a polynomial on the FMA pipe (228 to 243); two threads per pair (265 to 290); waits that spin (237 to 244).  What brought
// it from 480: registers for 64 scores instead of 128 without spilling, one lane that issues the copies (32 lanes with a copy each run one after
// the other), loops over the products unrolled.
#include <string.h>

#include "esp_attn_tc.cuh"
#include "esp_paged.cuh"

namespace esp {

namespace {

using namespace tc;
using namespace paged;

constexpr int CK = 128;                   // keys per chunk
constexpr int STEP = 64;                  // keys per step of the softmax: a chunk's halves one after the other
constexpr int SUB = 128;                  // pairs per subtile
constexpr int HALF_BYTES = 128 * 128;     // 128 rows x 64 elements, 128-byte swizzle
constexpr int THREADS = 384;
constexpr int TMEM_COLS = 512;            // S0, S1, O0, O1: 128 columns each
constexpr int ODD_RING = 8;               // pieces whose note on odd values is kept: the one being read, the next one, one for each stage of values, two that warp 3 enters

template <int D>
struct Cfg {
    static constexpr int HALVES = D / 64;
    static constexpr int TILE_BYTES = HALVES * HALF_BYTES;         // 128 rows of a head
    // Rings of their own for keys and values: whoever waits on a barrier has to see each of its phases and to be needed for the next one.  (With one
    // ring for both, whose stages held keys and values in turn, the warps that look at the values alone lost a phase once in a thousand calls.)
    static constexpr int KST = D == 128 ? 2 : 4, VST = D == 128 ? 3 : 4;
    static constexpr int OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + KST * TILE_BYTES;
    static constexpr int OFF_BAR = OFF_V + VST * TILE_BYTES;
    static constexpr int SMEM = 1024 + OFF_BAR + 512;
    // kind::f16 instruction descriptors: D = f32, A = B = bf16, M = 128; Q K^T: N = 128 keys; P V: N = D, V is MN-major
    static constexpr uint32_t IDESC_QK = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
    static constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
};

struct TcParams {
    CUtensorMap map_q;        // [tokens][heads][D], box 64 x group x rows of a subtile
    CUtensorMap map_k;        // [pages][heads][slots][D], box 64 x box_rows
    CUtensorMap map_v;
    PagedAttnArgs a;
    int32_t box_rows, sub_rows, out_vec;
};

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}
__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* map, int x, int y, int z) {
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global [%0, {%1, %2, %3}];" ::"l"(map), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ float max3_nan(float x, float y, float z) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(x), "f"(y), "f"(z));
    return d;
}
// The weights of a row's scores of one step, as bf16 over the scores' columns; their sum, of the weights before rounding.  bf16 is what one product with bf16 values takes: a
// weight is off by 2^-8 of itself at most, an output by 0.0023 of the norm instead of the 0.0017 that its own rounding costs.  Two products with hi + lo, as single tokens
// have them where memory is the bound, would be half as much tensor work again.
__device__ __forceinline__ float weights(const uint32_t (&sv)[STEP], uint32_t s_addr, float scale_log2, float m_use) {
    const uint64_t scale2 = attn::pack2(scale_log2, scale_log2), neg_m2 = attn::pack2(-m_use, -m_use);
    uint64_t sum2[2] = {0, 0};
    uint32_t pk[STEP / 2];
#pragma unroll
    for (int i = 0; i < STEP / 2; ++i) {
        float w0, w1;
        attn::unpack2(attn::fma2(attn::pack2(__uint_as_float(sv[2 * i]), __uint_as_float(sv[2 * i + 1])), scale2, neg_m2), w0, w1);
        w0 = attn::ex2_approx(w0);
        w1 = attn::ex2_approx(w1);
        sum2[i & 1] = attn::add2(sum2[i & 1], attn::pack2(w0, w1));
        const __nv_bfloat162 b2 = __floats2bfloat162_rn(w0, w1);
        pk[i] = *reinterpret_cast<const uint32_t*>(&b2);
    }
    tmem_st32(s_addr, pk);
    float c0, c1;
    attn::unpack2(attn::add2(sum2[0], sum2[1]), c0, c1);
    return c0 + c1;
}

// A tile of one subtile whose keys several CTAs share anyway, in a call with many chunks for each of them: its chunks go to the two sets of scores,
// accumulators and softmax warps in turn, each with a reference and a sum of its own, and the merge kernel joins one part more per
// CTA.  One set waits for every product and every softmax in turn; two parts cost the merge.  4 sequences of 16 tokens over 32k
// positions (54 chunks per CTA) 106 us with one set, 97 with two; 8 of 17 over 8k (28) 64 both; 32 of 4 over 4k (10) 61 and 63; 1 of 32 over 4k
// (2) 18 and 22.
__device__ __forceinline__ bool in_turn(const Piece& pc, int subs, const Share& share) { return subs == 1 && pc.slot >= 0 && share.each >= 32; }
__device__ __forceinline__ int chunks_of(const Piece& pc, int subs, int sub, const Share& share) { return in_turn(pc, subs, share) ? (pc.n + 1 - sub) / 2 : (sub < subs ? pc.n : 0); }

// A chunk that some pair of the tile does not see as a whole (the last one of the cache, the diagonal, the window's edge, the tree).
__device__ __forceinline__ bool is_edge(const PagedAttnArgs& a, const Cursor& c, int p0) {
    const int L = c.s.kv - c.s.n;
    const int hi = a.anc ? L : L + c.x.r0 + 1;
    const int lo = a.window > 0 ? L + c.x.r0 + c.x.nr - a.window : 0;
    return p0 + CK > hi || p0 < lo;
}
// the keys of the step at p0 as bits: which of them the pair sees
__device__ __forceinline__ void step_bits(const RowMask& m, int p0, int L, int n, uint32_t (&w)[2]) {
    const int lo = max(m.lo - p0, 0), hi = min(m.hi - p0, STEP);
    unsigned long long bits = hi > lo ? (hi - lo >= 64 ? ~0ull : ((1ull << (hi - lo)) - 1ull) << lo) : 0ull;
    if (m.b0 | m.b1) {
        // block row j stands at position L + j: bit j goes to bit j + L - p0
        unsigned long long b0 = m.b0, b1 = m.b1;
        if (n < 64) { b0 &= (1ull << n) - 1ull; b1 = 0; }
        else if (n < 128) b1 &= (1ull << (n - 64)) - 1ull;
        const int down = p0 - L;
        if (down == 0) bits |= b0;
        else if (down > 0 && down < 64) bits |= (b0 >> down) | (b1 << (64 - down));
        else if (down >= 64 && down < 128) bits |= b1 >> (down - 64);
        else if (down < 0 && down > -64) bits |= b0 << -down;
    }
    w[0] = (uint32_t)bits;
    w[1] = (uint32_t)(bits >> 32);
}

template <int D>
__global__ void __launch_bounds__(THREADS, 1) k_paged_tc(const __grid_constant__ TcParams p) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ int2 s_box[2][16];          // [keys, values] page and slot of a chunk's boxes
    __shared__ int s_odd[ODD_RING];        // a value that some pair sees is no finite number
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR); // [KST] keys of a chunk have landed
    uint64_t* k_empty = k_full + C::KST;                               // [KST] both subtiles' Q K^T have completed
    uint64_t* v_full = k_empty + C::KST;                               // [VST] values of a chunk have landed
    uint64_t* v_ok = v_full + C::VST;                                  // [VST] they have been looked after
    uint64_t* v_empty = v_ok + C::VST;                                 // [VST] both subtiles' P V have completed
    uint64_t* s_full = v_empty + C::VST;                               // [2] scores of a subtile's chunk
    uint64_t* p_ready = s_full + 2;                                    // [2][2] weights, by halves of the chunk
    uint64_t* pv_done = p_ready + 4;                                   // [2] the first half's P V has completed
    uint64_t* o_full = pv_done + 2;                                    // [2] the piece's last P V has completed
    uint64_t* o_free = o_full + 2;                                     // [2] the accumulator has been read
    uint64_t* q_full = o_free + 2;
    uint64_t* q_empty = q_full + 1;
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(q_empty + 1);
    volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);

    const PagedAttnArgs& a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        prefetch_tensormap(&p.map_k);
        prefetch_tensormap(&p.map_v);
        prefetch_tensormap(&p.map_q);
        for (int i = 0; i < C::KST; ++i) { mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 1); }
        for (int i = 0; i < C::VST; ++i) { mbar_init(&v_full[i], 1); mbar_init(&v_ok[i], 1); mbar_init(&v_empty[i], 1); }
        for (int i = 0; i < 4; ++i) mbar_init(&p_ready[i], 4);
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&pv_done[i], 1); mbar_init(&o_full[i], 1); mbar_init(&o_free[i], 4); }
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        *s_abort = 0;
        for (int i = 0; i < ODD_RING; ++i) s_odd[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    Share share;
    Cursor c;                              // every warp deals for itself and walks its own copy
    const bool any = deal<CK>(a, blockIdx.x, lane, share, c);
    const uint32_t begin = any ? share.begin(blockIdx.x) : 0, end = any ? share.begin(blockIdx.x + 1) : 0;
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = *s_tmem;
    unsigned char* sQ = smem;
    unsigned char *sK = smem + C::OFF_K, *sV = smem + C::OFF_V;

    if (warp == 0 || warp == 2) {
        // ---------------- TMA: warp 0 keys and queries, warp 2 values.  The lanes look up a chunk's pages, one lane issues box after box (a copy
        // issued by every lane for itself runs lane by lane, at some 50 cycles each)
        const bool is_v = warp == 2;
        const int n_boxes = CK / p.box_rows, box = lane & (n_boxes - 1);        // (a power of two: it divides the chunk)
        const CUtensorMap* map = is_v ? &p.map_v : &p.map_k;
        uint32_t ch = 0, n_it = 0;      // chunks, pieces
        bool ok = true;
        for (uint32_t u = begin; u < end && ok; ++n_it) {
            const Piece pc = make_piece(c, begin, u, end);
            for (int j = 0; j < pc.n; ++j, ++ch) {
                const int pos = (pc.c0 + j) * CK + box * p.box_rows;
                int page = a.pages.n_pages, slot = 0;       // a page that there is not reads as zeros
                if (pos < c.s.kv && pos + p.box_rows > first_seen(a, c.s, c.x.r0)) {
                    const int index = page_index(a.pages, pos);
                    const int pg = load_page(a.seq, a.pages, c.b, index);
                    if (pg >= 0) page = pg;
                    slot = pos - index * a.pages.page_size;
                }
                const uint32_t n_st = is_v ? C::VST : C::KST, st = ch % n_st;
                if (!__all_sync(0xffffffffu, mbar_wait((is_v ? v_empty : k_empty) + st, ((ch / n_st) & 1) ^ 1, s_abort))) { ok = false; break; }
                uint64_t* full = (is_v ? v_full : k_full) + st;
                if (lane == 0) mbar_expect_tx(full, C::TILE_BYTES);
                unsigned char* dst = (is_v ? sV : sK) + st * C::TILE_BYTES;
                if (lane < n_boxes) s_box[is_v][lane] = make_int2(page, slot);
                __syncwarp();
                if (lane == 0) {
#pragma unroll 4
                    for (int i = 0; i < n_boxes; ++i) {
                        const int2 b = s_box[is_v][i];
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h) tma_load_4d(dst + h * HALF_BYTES + i * p.box_rows * 128, map, h * 64, b.y, c.kvh, b.x, full);
                    }
                }
                if (!is_v && j == 0) {                      // the piece's queries behind its first keys
                    if (!__all_sync(0xffffffffu, mbar_wait(q_empty, (n_it & 1) ^ 1, s_abort))) { ok = false; break; }
                    if (lane == 0) {
                        const int subs = c.x.nr > p.sub_rows ? 2 : 1;
                        mbar_expect_tx(q_full, subs * C::HALVES * p.sub_rows * a.group * 128);
                        for (int s = 0; s < subs; ++s)
                            for (int h = 0; h < C::HALVES; ++h)
                                tma_load_3d(sQ + s * C::TILE_BYTES + h * HALF_BYTES, &p.map_q, h * 64, c.kvh * a.group, c.s.start + c.x.r0 + s * p.sub_rows, q_full);
                    }
                    if (u + pc.n < end) {                   // the next piece's queries come from far away: into L2 by then
                        Cursor nx = c;
                        next_tile<CK>(a, nx);
                        if (lane == 0)
                            for (int s = 0; s < (nx.x.nr > p.sub_rows ? 2 : 1); ++s)
                                for (int h = 0; h < C::HALVES; ++h) tma_prefetch_3d(&p.map_q, h * 64, nx.kvh * a.group, nx.s.start + nx.x.r0 + s * p.sub_rows);
                    }
                }
                __syncwarp();
            }
            u += pc.n;
            if (u < end) next_tile<CK>(a, c);
        }
        if (!ok && lane == 0) { set_error(a.seq.status, DEV_E_WAIT_TIMEOUT); *s_abort = 1; }
    } else if (warp == 1) {
        // ---------------- products: the warp walks its loop as a whole, one lane issues
        const bool leader{elect_lane()};
        const uint64_t q_desc = smem_desc(smem_u32(sQ), 16), k_desc = smem_desc(smem_u32(sK), 16), v_desc = smem_desc(smem_u32(sV), HALF_BYTES);
        uint32_t ch = 0, n_it = 0, g0 = 0, g1 = 0, pieces0 = 0, pieces1 = 0;   // chunks, pieces, chunks and pieces of each subtile
        bool ok = true;
        auto issue_qk = [&](int s, int q, int st) {          // scores s of the queries of subtile q
            const uint64_t da = q_desc + (uint32_t)(q * C::TILE_BYTES >> 4), db = k_desc + (uint32_t)(st * C::TILE_BYTES >> 4);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t off = ((kk >> 2) * HALF_BYTES + (kk & 3) * 32) >> 4;
                if (leader) umma(tmem_base + s * 128, da + off, db + off, C::IDESC_QK, kk > 0 ? 1u : 0u);
            }
            if (leader) umma_commit(&s_full[s]);
        };
        for (uint32_t u = begin; u < end && ok; ++n_it) {
            const Piece pc = make_piece(c, begin, u, end);
            const int subs = c.x.nr > p.sub_rows ? 2 : 1;
            const bool alt = in_turn(pc, subs, share);
            ok = __all_sync(0xffffffffu, mbar_wait(q_full, n_it & 1, s_abort) && mbar_wait(&k_full[ch % C::KST], (ch / C::KST) & 1, s_abort));
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (int s = 0; s < subs; ++s) issue_qk(s, s, ch % C::KST);
            if (leader) umma_commit(&k_empty[ch % C::KST]);
            const int ahead = alt ? 2 : 1;                               // a set of scores' next chunk
            if (alt && pc.n > 1) {
                ok = __all_sync(0xffffffffu, mbar_wait(&k_full[(ch + 1) % C::KST], ((ch + 1) / C::KST) & 1, s_abort));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                issue_qk(1, 0, (ch + 1) % C::KST);
                if (leader) umma_commit(&k_empty[(ch + 1) % C::KST]);
            }
            if (leader && pc.n <= ahead) umma_commit(q_empty);
            for (int j = 0; j < pc.n && ok; ++j, ++ch) {
                const uint32_t vs = ch % C::VST, kn = ch + ahead, ks = kn % C::KST;     // stages of this chunk's values, of the next keys
                const bool more = j + ahead < pc.n;
                const int jl = alt ? j >> 1 : j, s_end = alt ? (j & 1) + 1 : subs;
#pragma unroll 1
                for (int s = alt ? j & 1 : 0; s < s_end; ++s) {
                    const uint32_t g = s ? g1 : g0, np = s ? pieces1 : pieces0;
                    const uint64_t db = v_desc + (uint32_t)(vs * C::TILE_BYTES >> 4);
                    const uint32_t pa = tmem_base + s * 128;
                    const bool first = alt || s == 0;
                    // the first half of the weights, as soon as it stands
                    ok = __all_sync(0xffffffffu, (!first || mbar_wait(&v_ok[vs], (ch / C::VST) & 1, s_abort)) &&
                                                     (jl > 0 || mbar_wait(&o_free[s], (np & 1) ^ 1, s_abort)) && mbar_wait(&p_ready[2 * s], (g + jl) & 1, s_abort));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int kk = 0; kk < STEP / 16; ++kk)
                        if (leader) umma_ta(pa + 256, pa + kk * 8, db + (kk * 16 * 128 >> 4), C::IDESC_PV, (jl + kk > 0) ? 1u : 0u);
                    if (leader) umma_commit(&pv_done[s]);
                    ok = __all_sync(0xffffffffu, (!first || !more || mbar_wait(&k_full[ks], (kn / C::KST) & 1, s_abort)) &&
                                                     mbar_wait(&p_ready[2 * s + 1], (g + jl) & 1, s_abort));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int kk = STEP / 16; kk < CK / 16; ++kk)
                        if (leader) umma_ta(pa + 256, pa + STEP / 2 + kk * 8, db + (kk * 16 * 128 >> 4), C::IDESC_PV, 1u);
                    if (more) issue_qk(s, alt ? 0 : s, ks);
                    else if (leader) umma_commit(&o_full[s]);
                    if (leader && s == s_end - 1) {
                        umma_commit(&v_empty[vs]);
                        if (more) umma_commit(&k_empty[ks]);
                        if (j + ahead + 1 == pc.n) umma_commit(q_empty);
                    }
                }
            }
            const int n1 = chunks_of(pc, subs, 1, share);
            // subtile 1 may rest for any number of pieces: the last one it had has to have been read, or the ring of s_odd could come round
            if (ok && n1 == 0) ok = __all_sync(0xffffffffu, mbar_wait(&o_free[1], (pieces1 & 1) ^ 1, s_abort));
            g0 += chunks_of(pc, subs, 0, share);
            ++pieces0;
            g1 += n1;
            pieces1 += n1 > 0;
            u += pc.n;
            if (u < end) next_tile<CK>(a, c);
        }
        if (!ok && lane == 0) { set_error(a.seq.status, DEV_E_WAIT_TIMEOUT); *s_abort = 1; }
    } else if (warp == 3) {
        // ---------------- values: in chunks that not every pair sees, what is no finite number becomes zero before the product
        uint32_t ch = 0, n_it = 0;
        bool ok = true;
        Descs desc;
        desc.clear();
        for (uint32_t u = begin; u < end && ok; ++n_it) {
            const Piece pc = make_piece(c, begin, u, end);
            desc.note(a, c, share, pc, in_turn(pc, c.x.nr > p.sub_rows ? 2 : 1, share));
            if (lane == 0) s_odd[(n_it + 1) % ODD_RING] = 0;
            for (int j = 0; j < pc.n; ++j, ++ch) {
                const int st = ch % C::VST, p0 = (pc.c0 + j) * CK;
                if (!__all_sync(0xffffffffu, mbar_wait(&v_full[st], (ch / C::VST) & 1, s_abort))) { ok = false; break; }
                if (is_edge(a, c, p0)) {
                    uint4* tile = reinterpret_cast<uint4*>(sV + st * C::TILE_BYTES);
                    uint32_t seen = 0;          // an exponent of all ones carries into its sign bit
#pragma unroll 8
                    for (int i = lane; i < C::TILE_BYTES / 16; i += 32) {
                        const uint4 x = tile[i];
                        seen |= ((x.x & 0x7f807f80u) + 0x00800080u) | ((x.y & 0x7f807f80u) + 0x00800080u) | ((x.z & 0x7f807f80u) + 0x00800080u) |
                                ((x.w & 0x7f807f80u) + 0x00800080u);
                    }
                    bool odd = false;
                    if (seen & 0x80008000u) {
                        for (int i = lane; i < C::TILE_BYTES / 16; i += 32) {
                            uint4 x = tile[i];
                            uint32_t* w = reinterpret_cast<uint32_t*>(&x);
                            bool here = false;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; here = true; }
                                if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0x0000ffffu; here = true; }
                            }
                            if (here) {
                                tile[i] = x;
                                odd = odd || p0 + ((i >> 3) & 127) < c.s.kv;
                            }
                        }
                    }
                    if (odd) s_odd[n_it % ODD_RING] = 1;
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                if (lane == 0) mbar_arrive(&v_ok[st]);
            }
            u += pc.n;
            if (u < end) next_tile<CK>(a, c);
        }
        if (lane == 0) desc.store(a, blockIdx.x);
        if (!ok && lane == 0) { set_error(a.seq.status, DEV_E_WAIT_TIMEOUT); *s_abort = 1; }
    } else {
        // ---------------- softmax and output of subtile sub: a thread per pair
        const int sub = (warp - 4) >> 2, q4 = warp & 3, row = q4 * 32 + lane;
        const uint32_t s_addr = tmem_base + ((uint32_t)(q4 * 32) << 16) + sub * 128, o_addr = s_addr + 256;
        uint32_t g = 0, np = 0, n_it = 0;
        bool ok = true;
        for (uint32_t u = begin; u < end && ok; ++n_it) {
            const Piece pc = make_piece(c, begin, u, end);
            const int L = c.s.kv - c.s.n;
            const int subs = c.x.nr > p.sub_rows ? 2 : 1, n_mine = chunks_of(pc, subs, sub, share);
            const bool alt = in_turn(pc, subs, share);
            if (n_mine > 0) {
                const int pair = (alt ? 0 : sub * p.sub_rows * a.group) + row;   // of the tile
                const int part_pair = alt ? sub * SUB + row : pair;              // where its split partial goes
                const bool valid = row < p.sub_rows * a.group && pair < c.x.nr * a.group;
                const int trow = pair / a.group, head = c.kvh * a.group + pair - trow * a.group;
                RowMask mask;                  // (a lane without a pair may see anything: nobody reads its row)
                mask.lo = 0;
                mask.hi = KV_LIMIT;
                mask.b0 = mask.b1 = 0;
                if (valid) mask = row_mask(a, c.s, c.x.r0 + trow);
                const bool live = __any_sync(0xffffffffu, valid);
                float m_run = -INFINITY, l_run = 0.f;
#pragma unroll 2                                                                 // (the two halves as code of their own: 220 us, as a loop 245)
                for (int i = 0; i < 2 * n_mine; ++i) {
                    const int h = i & 1;                                         // half h of a chunk goes through half h of the columns
                    const uint32_t gc = g + (i >> 1);                            // chunks of this subtile so far
                    // (a wait that fails takes the whole warp out: the accesses to tensor memory are warp-wide)
                    if (h == 0) {
                        if (!__all_sync(0xffffffffu, mbar_wait(&s_full[sub], gc & 1, s_abort))) { ok = false; break; }
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    }
                    if (live) {
                        const int p0 = (pc.c0 + (alt ? 2 * (i >> 1) + sub : i >> 1)) * CK + h * STEP;
                        uint32_t sv[STEP];
                        attn::tmem_ld64(s_addr + h * STEP, sv);
                        const bool whole = __all_sync(0xffffffffu, p0 >= mask.lo && p0 + STEP <= mask.hi);
                        if (!whole) {
                            uint32_t w[2];
                            step_bits(mask, p0, L, c.s.n, w);
#pragma unroll
                            for (int e = 0; e < STEP; ++e) sv[e] = (w[e >> 5] >> (e & 31)) & 1u ? sv[e] : 0xff800000u;
                        }
                        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int e = 0; e < STEP; e += 8)
#pragma unroll
                            for (int f = 0; f < 4; ++f) m4[f] = max3_nan(m4[f], __uint_as_float(sv[e + 2 * f]), __uint_as_float(sv[e + 2 * f + 1]));
                        float cmax = max3_nan(m4[0], m4[1], max3_nan(m4[2], m4[3], m4[3])) * a.scale_log2;
                        // a logit that is no number or +infinity makes the whole row undefined, and so does a reference that is no number
                        if (!(cmax < INFINITY)) cmax = __int_as_float(0x7fffffff);
                        const bool move = m_run == -INFINITY ? cmax != -INFINITY : !(cmax - m_run <= 8.f);
                        const float m_new = move ? cmax : m_run;
                        const float m_use = m_new == -INFINITY ? 0.f : m_new;
                        float alpha = 1.f;
                        if (__any_sync(0xffffffffu, move)) alpha = m_run == m_use ? 1.f : exp2f(m_run - m_use);
                        const float csum = weights(sv, s_addr + h * STEP, a.scale_log2, m_use);
                        l_run = fmaf(l_run, alpha, csum);
                        m_run = m_new;
                        if (i > 0 && __any_sync(0xffffffffu, move)) {
                            // O <- O * 2^(old - new).  The chunk's scores said that the products of the chunk before have completed; within a chunk the
                            // first half's has to.  (Its phase before is over for the same reason, and the next one waits for this half's weights: no
                            // phase can be mistaken for another.)
                            if (h == 1) {
                                if (!__all_sync(0xffffffffu, mbar_wait(&pv_done[sub], gc & 1, s_abort))) { ok = false; break; }
                                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                            }
#pragma unroll 1
                            for (int b = 0; b < D / 32; ++b) {
                                uint32_t o[32];
                                tmem_ld32(o_addr + b * 32, o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                                tmem_st32(o_addr + b * 32, o);
                            }
                        }
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    }
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_ready[2 * sub + h]);
                }
                g += n_mine;
                if (!ok) break;
                if (!__all_sync(0xffffffffu, mbar_wait(&o_full[sub], np & 1, s_abort))) { ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                ++np;
                if (live) {
                    const bool odd = *reinterpret_cast<volatile int*>(&s_odd[n_it % ODD_RING]) != 0;
                    const int token = c.s.start + c.x.r0 + trow;
                    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
#pragma unroll 1
                    for (int b = 0; b < D / 32; ++b) {
                        uint32_t o[32];
                        tmem_ld32(o_addr + b * 32, o);
                        if (odd && valid) {
                            // the values that were set to zero, for the pairs that see them
                            for (int j = alt ? sub : 0; j < pc.n; j += alt ? 2 : 1) {
                                const int p0 = (pc.c0 + j) * CK;
                                if (!is_edge(a, c, p0)) continue;
                                for (int pos = p0; pos < min(p0 + CK, c.s.kv); ++pos) {
                                    if (!sees(mask, pos, L, c.s.kv)) continue;
                                    const int index = page_index(a.pages, pos);
                                    const int page = load_page(a.seq, a.pages, c.b, index);
                                    if (page < 0) continue;
                                    const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(a.pages.v) + page * a.pages.page +
                                                             (pos - index * a.pages.page_size) * a.pages.tok + c.kvh * a.pages.head + b * 32;
#pragma unroll
                                    for (int i = 0; i < 32; ++i) {
                                        const float x = to_f32(v[i]);
                                        if (!isfinite(x)) o[i] = __float_as_uint(__uint_as_float(o[i]) + x);
                                    }
                                }
                            }
                        }
                        if (valid && pc.slot < 0) {
                            __nv_bfloat16* y = reinterpret_cast<__nv_bfloat16*>(a.out.p) + out_offset(a.out, token, head) + b * 32;
                            uint32_t pk[16];
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const __nv_bfloat162 b2 = __floats2bfloat162_rn(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv);
                                pk[i >> 1] = *reinterpret_cast<const uint32_t*>(&b2);
                            }
                            if (p.out_vec) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(y + i * 8) = make_uint4(pk[4 * i], pk[4 * i + 1], pk[4 * i + 2], pk[4 * i + 3]);
                            } else {
#pragma unroll
                                for (int i = 0; i < 32; ++i) y[i] = __ushort_as_bfloat16((unsigned short)(pk[i >> 1] >> ((i & 1) * 16)));
                            }
                        } else if (valid) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                *reinterpret_cast<uint4*>(a.part_o + part_quad(a, blockIdx.x, pc.slot, b * 8 + i, part_pair)) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                        }
                    }
                    if (valid && pc.slot >= 0) a.part_ml[part_row(a, blockIdx.x, pc.slot, part_pair)] = make_float2(m_run, l_run);
                    if (valid && pc.slot < 0 && a.lse) a.lse[(size_t)token * a.Hq + head] = l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * 0.6931471805599453f;
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&o_free[sub]);
            } else if (alt) {
                a.part_ml[part_row(a, blockIdx.x, pc.slot, sub * SUB + row)] = make_float2(-INFINITY, 0.f);       // one chunk only: nothing left for this set
            }
            u += pc.n;
            if (u < end) next_tile<CK>(a, c);
        }
        if (!ok && lane == 0) { set_error(a.seq.status, DEV_E_WAIT_TIMEOUT); *s_abort = 1; }
    }
    // ---------------- teardown (every thread arrives here)
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (*s_abort) {
        for (int i = 0; i < 64; ++i) __nanosleep(10000);   // let copies in flight land before shared memory goes away
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS) : "memory");
    }
}

int gcd(int x, int y) { return y ? gcd(y, x % y) : x; }

template <int D>
int run_tc(TcParams& p, cudaStream_t s) {
    if (ensure_dynamic_smem(reinterpret_cast<const void*>(&k_paged_tc<D>), Cfg<D>::SMEM)) return -1;
    k_paged_tc<D><<<p.a.n_cta, THREADS, Cfg<D>::SMEM, s>>>(p);
    return 0;
}

}  // namespace

bool paged_tma_pages(const PagedAttnArgs& a, int chunk, int* box_rows) {
    // boxes of whole swizzle groups of eight rows; every stride a multiple of 16 bytes below 2^40
    *box_rows = gcd(a.pages.page_size, chunk);
    auto al = [](long long x) { return x % 8 == 0 && x < (1ll << 39); };
    return *box_rows % 8 == 0 && reinterpret_cast<uintptr_t>(a.pages.k) % 16 == 0 && reinterpret_cast<uintptr_t>(a.pages.v) % 16 == 0 && al(a.pages.page) &&
           al(a.pages.tok) && al(a.pages.head) && a.pages.page_size <= (1 << 30);
}
int paged_page_map(CUtensorMap* map, const PagedAttnArgs& a, const void* base, int box_rows) {
    EncodeFn enc = get_encode();
    if (!enc) return -1;
    auto bytes = [&](long long stride) { return (cuuint64_t)(stride > 0 ? stride * 2 : a.D * 2); };      // (a dimension of one element: any stride)
    cuuint64_t dims[4] = {(cuuint64_t)a.D, (cuuint64_t)a.pages.page_size, (cuuint64_t)a.Hkv, (cuuint64_t)a.pages.n_pages};
    cuuint64_t strides[3] = {bytes(a.pages.tok), bytes(a.pages.head), bytes(a.pages.page)};
    cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? 0 : -1;
}

bool paged_tc_supported(int dtype, const PagedAttnArgs& a) {
    int box = 0;
    return dtype == 1 && (a.D == 64 || a.D == 128) && a.group <= SUB && paged_tma_pages(a, CK, &box) && reinterpret_cast<uintptr_t>(a.q.p) % 16 == 0 &&
           a.q.tok % 8 == 0 && a.q.head % 8 == 0 && a.q.tok < (1ll << 39) && a.q.head < (1ll << 39) && (a.q.tok > 0 || a.seq.n_tokens == 1) && (a.q.head > 0 || a.Hq == 1);
}

int launch_paged_tc(PagedAttnArgs a, int n_sm, cudaStream_t s) {
    TcParams p;
    memset(&p, 0, sizeof(p));
    if (!paged_tma_pages(a, CK, &p.box_rows)) return -1;
    if (paged_page_map(&p.map_k, a, a.pages.k, p.box_rows) || paged_page_map(&p.map_v, a, a.pages.v, p.box_rows)) return -1;
    p.sub_rows = SUB / a.group;
    {
        EncodeFn enc = get_encode();
        cuuint64_t dims[3] = {(cuuint64_t)a.D, (cuuint64_t)a.Hq, (cuuint64_t)a.seq.n_tokens};
        cuuint64_t strides[2] = {(cuuint64_t)(a.q.head > 0 ? a.q.head * 2 : a.D * 2), (cuuint64_t)(a.q.tok > 0 ? a.q.tok * 2 : a.D * 2)};
        cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)p.sub_rows};
        const cuuint32_t estr[3] = {1, 1, 1};
        if (enc(&p.map_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, a.q.p, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) return -1;
    }
    a.rows = 2 * p.sub_rows;
    a.rows_shift = shift_of(a.rows);
    a.pairs = 2 * SUB;
    a.n_cta = n_sm;
    p.out_vec = reinterpret_cast<uintptr_t>(a.out.p) % 16 == 0 && a.out.tok % 8 == 0 && a.out.head % 8 == 0;
    p.a = a;
    const int rc = a.D == 128 ? run_tc<128>(p, s) : run_tc<64>(p, s);
    return rc ? rc : launch_paged_merge(1, a, s);
}

}  // namespace esp
