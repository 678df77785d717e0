// Weights of cached positions on the Blackwell tensor cores: bf16, heads of 64 or 128, blocks of several tokens.
//
// A CTA holds a chunk of 256 keys in shared memory, as two subtiles of 128, and walks the tiles of up to 128 (token, query head) pairs that see it:
//   S_s = K_s Q^T    tcgen05.mma with the keys as rows, both operands K-major in shared memory, 128 x 128 fp32 in tensor memory, two sets of both subtiles;
//   weights          two threads per key (= tensor-memory lane), for a half of the columns each: exp(scale s - lse), added up in a register; a mask is a range of columns.
// So a key's sum never leaves its thread while the chunk stays, keys are read once and queries once for every 256 keys.
// What bounds it: one exponential a pair and key, 2048 cycles of an SM's special-function units for 256 keys and 128 pairs, twice what the products take.  2048 tokens at
// the end of 8192, 32/8 heads of 128: 2750 cycles a tile, 165 us (71 us of products at the cuBLAS rate).  Built and slower (us there): 8 warps of weights 190; a part of the
// exponentials as polynomials 175 to 188 (an eighth to a half of them; what they cost was not looked into: the kernel uses 39 % of its issue slots); the two groups of warps on alternate tiles
// 179; masks by comparing every column 170.  For few tiles the start counts: 64 tokens of one sequence took 22 us with one warp issuing the keys' boxes, 17.5 with two.
// Roles: warps 0 and 3 TMA (a subtile's keys each, warp 0 the queries too), warp 1 issues the products, warp 2 brings the tiles' lse, warps 4-19 have the weights.  Every wait is bounded; one
// that runs out is recorded, the tensor memory is given back and the kernel returns.
#include <string.h>

#include "esp_attn_tc.cuh"
#include "esp_key_weights.cuh"

namespace esp {

namespace {

using namespace tc;
using namespace paged;

constexpr int CK = KEY_WEIGHT_KEYS, SUB = 128, PAIRS = 128;
constexpr int HALF_BYTES = 128 * 128;     // 128 rows x 64 elements, 128-byte swizzle
constexpr int SUM_WARPS = 16, THREADS = 128 + SUM_WARPS * 32;
constexpr int TMEM_COLS = 512;            // [set][subtile][128]

template <int D>
struct Cfg {
    static constexpr int HALVES = D / 64;
    static constexpr int TILE_BYTES = HALVES * HALF_BYTES;         // 128 rows of a head
    static constexpr int KST = D == 128 ? 2 : 3, QST = D == 128 ? 2 : 4, LST = 4;      // (even: a tile of every other chunk has its own places)
    static constexpr int OFF_Q = KST * 2 * TILE_BYTES, OFF_LSE = OFF_Q + QST * TILE_BYTES, OFF_HALF = OFF_LSE + LST * PAIRS * 4, OFF_BAR = OFF_HALF + CK * 4;
    static constexpr int SMEM = 1024 + OFF_BAR + 512;
    // kind::f16 instruction descriptor: D = f32, A = B = bf16, M = 128, N = 128
    static constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
};

struct TcParams {
    CUtensorMap map_q;        // [tokens][heads][D], box 64 x group x rows of a tile
    CUtensorMap map_k;        // [pages][heads][slots][D], box 64 x box_rows
    KeyWeightArgs w;
    int32_t box_rows, group_inv;      // group_inv: 2^16 / group, rounded up (column / group for columns below 128)
};

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}

// acc + 2^x of a pair
__device__ __forceinline__ uint64_t exp_add(uint64_t x, uint64_t acc) {
    float x0, x1;
    attn::unpack2(x, x0, x1);
    return attn::add2(acc, attn::pack2(attn::ex2_approx(x0), attn::ex2_approx(x1)));
}
// ONE: no sequence has more observed tokens than a tile.
template <int D, bool ONE>
__global__ void __launch_bounds__(THREADS, 1) k_key_weights_tc(const __grid_constant__ TcParams p) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ int2 s_box[2][16];          // [subtile] page and slot of a chunk's boxes
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char *sK = smem, *sQ = smem + C::OFF_Q;
    float* s_lse = reinterpret_cast<float*>(smem + C::OFF_LSE);        // [LST][PAIRS] -lse in the log2 domain
    float* s_half = reinterpret_cast<float*>(smem + C::OFF_HALF);      // [CK] sums over the second half of the columns
    uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR); // [KST] keys of a chunk have landed
    uint64_t* k_empty = k_full + C::KST;                               // [KST] their last product has completed
    uint64_t* q_full = k_empty + C::KST;                               // [QST] queries of a tile have landed
    uint64_t* q_empty = q_full + C::QST;                               // [QST] its products have completed
    uint64_t* l_full = q_empty + C::QST;                               // [LST] a tile's lse stand (a ring of their own: the queries' places are free a tile earlier)
    uint64_t* l_empty = l_full + C::LST;                               // [LST] they have been read
    uint64_t* s_full = l_empty + C::LST;                               // [2] scores of a set
    uint64_t* s_free = s_full + 2;                                     // [2] they have been read
    uint64_t* h_full = s_free + 2;                                     // [8] the second half's sums of 32 keys stand
    uint64_t* h_free = h_full + 8;                                     // [8] they have been taken
    uint32_t* s_tmem = reinterpret_cast<uint32_t*>(h_free + 8);
    volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);

    const KeyWeightArgs& w = p.w;
    const PagedAttnArgs& a = w.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        prefetch_tensormap(&p.map_k);
        prefetch_tensormap(&p.map_q);
        for (int i = 0; i < C::KST; ++i) { mbar_init(&k_full[i], 2); mbar_init(&k_empty[i], 1); }
        for (int i = 0; i < C::QST; ++i) { mbar_init(&q_full[i], 1); mbar_init(&q_empty[i], 1); }
        for (int i = 0; i < C::LST; ++i) { mbar_init(&l_full[i], 1); mbar_init(&l_empty[i], ONE ? SUM_WARPS / 2 : SUM_WARPS); }
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&s_free[i], ONE ? SUM_WARPS / 2 : SUM_WARPS); }
        for (int i = 0; i < 8; ++i) { mbar_init(&h_full[i], 1); mbar_init(&h_free[i], 1); }
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(s_tmem)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_launch_dependents();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    Share share;
    WCursor c;                             // every warp deals for itself and walks its own copy
    const bool any = deal_keys<CK>(w, blockIdx.x, lane, share, c);
    const uint32_t begin = any ? share.begin(blockIdx.x) : 0, end = any ? share.begin(blockIdx.x + 1) : 0;
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = *s_tmem;

    if (warp == 0 || warp == 3) {
        // ---------------- TMA: the lanes look up a chunk's pages, one lane issues box after box; warp 0 has the first subtile's and the queries, warp 3 the second's
        const int sub = warp == 3, n_boxes = SUB / p.box_rows;       // a power of two, 16 at most
        uint32_t n_k = 0, n_q = 0;                  // chunks and tiles so far
        bool ok = true;
        for (uint32_t u = begin; u < end && ok;) {
            const WPiece pc = make_piece(c, begin, u, end);
            if (pc.n > 0) {
                const int pos = c.c * CK + sub * SUB + (lane & (n_boxes - 1)) * p.box_rows;
                int page = a.pages.n_pages, slot = 0;       // a page that there is not reads as zeros
                if (pos < c.x.s.kv && pos + p.box_rows > first_observed(w, c.x)) {
                    const int index = page_index(a.pages, pos);
                    const int pg = load_page(a.seq, a.pages, c.b, index);
                    if (pg >= 0) page = pg;
                    slot = pos - index * a.pages.page_size;
                }
                const uint32_t st = n_k % C::KST;
                if (!__all_sync(0xffffffffu, mbar_wait(&k_empty[st], ((n_k / C::KST) & 1) ^ 1, s_abort))) { ok = false; break; }
                if (lane < n_boxes) s_box[sub][lane] = make_int2(page, slot);
                __syncwarp();
                if (lane == 0) {
                    mbar_expect_tx(&k_full[st], C::TILE_BYTES);
                    unsigned char* dst = sK + (st * 2 + sub) * C::TILE_BYTES;
                    for (int i = 0; i < n_boxes; ++i) {
                        const int2 b = s_box[sub][i];
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h) tma_load_4d(dst + i * p.box_rows * 128 + h * HALF_BYTES, &p.map_k, h * 64, b.y, c.kvh, b.x, &k_full[st]);
                    }
                }
                __syncwarp();
                ++n_k;
                for (int t = pc.t0; t < pc.t0 + pc.n && sub == 0; ++t, ++n_q) {
                    const uint32_t sq = n_q % C::QST;
                    if (!__all_sync(0xffffffffu, mbar_wait(&q_empty[sq], ((n_q / C::QST) & 1) ^ 1, s_abort))) { ok = false; break; }
                    if (lane == 0) {
                        mbar_expect_tx(&q_full[sq], C::HALVES * a.rows * a.group * 128);
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h)
                            tma_load_3d(sQ + sq * C::TILE_BYTES + h * HALF_BYTES, &p.map_q, h * 64, c.kvh * a.group, c.x.s.start + c.x.i0 + t * a.rows, &q_full[sq]);
                    }
                    __syncwarp();
                }
            }
            u += max(pc.n, 1);
            if (u < end) next_chunk<CK>(w, c);
        }
        if (!ok && lane == 0) { set_error(a.seq.status, DEV_E_WAIT_TIMEOUT); *s_abort = 1; }
    } else if (warp == 1) {
        // ---------------- products: the warp walks its loop as a whole, one lane issues
        const bool leader{elect_lane()};
        const uint64_t k_desc = smem_desc(smem_u32(sK), 16), q_desc = smem_desc(smem_u32(sQ), 16);
        uint32_t n_k = 0, n = 0;                    // chunks and tiles so far
        bool ok = true;
        for (uint32_t u = begin; u < end && ok;) {
            const WPiece pc = make_piece(c, begin, u, end);
            if (pc.n > 0) {
                const uint32_t st = n_k % C::KST;
                ok = __all_sync(0xffffffffu, mbar_wait(&k_full[st], (n_k / C::KST) & 1, s_abort));
                if (!ok) break;
                for (int t = 0; t < pc.n; ++t, ++n) {
                    const uint32_t sq = n % C::QST, set = n & 1;
                    ok = __all_sync(0xffffffffu, mbar_wait(&q_full[sq], (n / C::QST) & 1, s_abort) && mbar_wait(&s_free[set], ((n >> 1) & 1) ^ 1, s_abort));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t db = q_desc + (uint32_t)(sq * C::TILE_BYTES >> 4);
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const uint64_t da = k_desc + (uint32_t)((st * 2 + s) * C::TILE_BYTES >> 4);
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint32_t off = ((kk >> 2) * HALF_BYTES + (kk & 3) * 32) >> 4;
                            if (leader) umma(tmem_base + set * 256 + s * 128, da + off, db + off, C::IDESC, kk > 0 ? 1u : 0u);
                        }
                    }
                    if (leader) umma_commit(&s_full[set]);
                    if (leader) umma_commit(&q_empty[sq]);
                }
                if (!ok) break;
                if (leader) umma_commit(&k_empty[st]);
                ++n_k;
            }
            u += max(pc.n, 1);
            if (u < end) next_chunk<CK>(w, c);
        }
        if (!ok && lane == 0) { set_error(a.seq.status, DEV_E_WAIT_TIMEOUT); *s_abort = 1; }
    } else if (warp == 2) {
        // ---------------- lse of the tiles' pairs
        uint32_t n = 0;
        bool ok = true;
        for (uint32_t u = begin; u < end && ok;) {
            const WPiece pc = make_piece(c, begin, u, end);
            for (int t = pc.t0; t < pc.t0 + pc.n; ++t, ++n) {
                const int r0 = c.x.i0 + t * a.rows, pairs = min(a.rows, c.x.s.n - r0) * a.group;
                float x[PAIRS / 32];
#pragma unroll
                for (int j = 0; j < PAIRS / 32; ++j) {
                    const int col = j * 32 + lane, row = (col * p.group_inv) >> 16;
                    x[j] = col < pairs ? __ldg(w.lse + (size_t)(c.x.s.start + r0 + row) * a.Hq + c.kvh * a.group + col - row * a.group) * -1.4426950408889634f : 0.f;
                }
                const uint32_t sl = n % C::LST;
                if (!__all_sync(0xffffffffu, mbar_wait(&l_empty[sl], ((n / C::LST) & 1) ^ 1, s_abort))) { ok = false; break; }
#pragma unroll
                for (int j = 0; j < PAIRS / 32; ++j) s_lse[sl * PAIRS + j * 32 + lane] = x[j];
                __syncwarp();
                if (lane == 0) mbar_arrive(&l_full[sl]);
            }
            u += max(pc.n, 1);
            if (u < end) next_chunk<CK>(w, c);
        }
        if (!ok && lane == 0) { set_error(a.seq.status, DEV_E_WAIT_TIMEOUT); *s_abort = 1; }
    } else if (warp >= 4) {
        // ---------------- weights.  warps 4-7 and 8-11 (the first of two halves) have the subtiles' first 64 columns, 12-15 and 16-19 the others; where no chunk meets more
        // than one tile (ONE), the first half of the warps has every other chunk as a whole: nothing is put together, and one chunk's loads and stores fall into the other's exponentials
        const int sub = ((warp - 4) >> 2) & 1, half = (warp - 4) >> 3, pair = sub * 4 + (warp & 3), key = pair * 32 + lane;
        const uint32_t s_addr = tmem_base + sub * 128 + ((uint32_t)((warp & 3) * 32) << 16);
        const int col0 = ONE ? 0 : half * 64;
        uint32_t n = 0, n_p = 0;
        bool ok = true;
        for (uint32_t u = begin; u < end && ok; ++n_p) {
            const WPiece pc = make_piece(c, begin, u, end);
            const Seq s = c.x.s;
            const int L = s.kv - s.n, p0 = c.c * CK, pos = p0 + key;
            const bool mine = !ONE || (pc.n > 0 ? (int)(n & 1) == half : half == 0);
            const bool writes = ONE ? mine : half == 0;
            // the place of the score, and what it holds, before the weights are there
            float *to = nullptr, old = 0.f;
            if (writes && pc.slot < 0 && pos < s.kv) {
                to = score_at(w, c, pos);
                if (to && has_old(w, s, pos)) old = *to;
            }
            float sum0 = 0.f;
            uint64_t acc_a = 0, acc_b = 0;
            for (int t = pc.t0; t < pc.t0 + pc.n; ++t, ++n) {
                if (!mine) continue;
                const uint32_t sl = n % C::LST, set = n & 1;
                const int r0 = c.x.i0 + t * a.rows, nr = min(a.rows, s.n - r0);
                // columns that see this key: all pairs of the tile, or a range of its tokens, or, inside the block of a tree, as their masks say
                int lo = 0, hi = nr * a.group;
                bool tree = false;
                const bool edge = hi < PAIRS || p0 + CK > (a.anc ? L : L + r0 + 1) || (a.window > 0 && p0 < L + r0 + nr - a.window);
                if (edge) {
                    if (pos >= s.kv) hi = 0;
                    else if (a.anc) {
                        if (pos >= L) tree = true;
                        else if (L + r0 < 0) lo = min(nr, -(L + r0)) * a.group;            // padding sees nothing
                    } else {
                        lo = min(max(pos - L - r0, 0), nr) * a.group;
                        if (a.window > 0) hi = (int)min(max((long long)pos - L + a.window - r0, 0ll), (long long)nr) * a.group;
                    }
                }
                ok = __all_sync(0xffffffffu, mbar_wait(&l_full[sl], (n / C::LST) & 1, s_abort) && mbar_wait(&s_full[set], (n >> 1) & 1, s_abort));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const float4* nl = reinterpret_cast<const float4*>(s_lse + sl * PAIRS + col0);
#pragma unroll 1
                for (int b = 0; b < (ONE ? 4 : 2); ++b) {
                    uint32_t y[32];
                    tmem_ld32(s_addr + set * 256 + col0 + b * 32, y);
                    if (!edge) {
                        const uint64_t scale2 = attn::pack2(a.scale_log2, a.scale_log2);
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 m = nl[b * 8 + j / 4];
                            acc_a = exp_add(attn::fma2(attn::pack2(__uint_as_float(y[j]), __uint_as_float(y[j + 1])), scale2, attn::pack2(m.x, m.y)), acc_a);
                            acc_b = exp_add(attn::fma2(attn::pack2(__uint_as_float(y[j + 2]), __uint_as_float(y[j + 3])), scale2, attn::pack2(m.z, m.w)), acc_b);
                        }
                    } else if (!__any_sync(0xffffffffu, tree)) {
                        const int l = lo - col0 - b * 32, r = hi - col0 - b * 32;
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 m = nl[b * 8 + j / 4];
                            const float mm[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float v = attn::ex2_approx(fmaf(__uint_as_float(y[j + e]), a.scale_log2, mm[e]));
                                sum0 += j + e >= l && j + e < r ? v : 0.f;
                            }
                        }
                    } else {
                        const int bit = min(max(pos - L, 0), 127);
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const int col = col0 + b * 32 + j, i = r0 + ((col * p.group_inv) >> 16);
                            bool in = col >= lo && col < hi;
                            if (tree && in)
                                in = L + i >= 0 && pos - L < 128 && ((__ldg(a.anc + 2 * (size_t)(s.start + i) + (bit >> 6)) >> (bit & 63)) & 1);
                            const float v = attn::ex2_approx(fmaf(__uint_as_float(y[j]), a.scale_log2, reinterpret_cast<const float*>(nl)[b * 32 + j]));
                            sum0 += in ? v : 0.f;
                        }
                    }
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&s_free[set]);
                    mbar_arrive(&l_empty[sl]);
                }
            }
            if (!ok) break;
            float sa0, sa1, sb0, sb1;
            attn::unpack2(acc_a, sa0, sa1);
            attn::unpack2(acc_b, sb0, sb1);
            float sum = sum0 + ((sa0 + sa1) + (sb0 + sb1));
            if (!ONE) {                                          // the halves' sums together
                if (half == 1) {
                    ok = __all_sync(0xffffffffu, mbar_wait(&h_free[pair], (n_p & 1) ^ 1, s_abort));
                    if (!ok) break;
                    s_half[key] = sum;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&h_full[pair]);
                } else {
                    ok = __all_sync(0xffffffffu, mbar_wait(&h_full[pair], n_p & 1, s_abort));
                    if (!ok) break;
                    sum += s_half[key];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&h_free[pair]);
                    if (pc.slot >= 0) w.part[((size_t)blockIdx.x * 2 + pc.slot) * KEY_WEIGHT_KEYS + key] = sum;
                }
            }
            if (to) *to = has_old(w, s, pos) ? fmaf(w.keep, old, sum) : sum;
            u += max(pc.n, 1);
            if (u < end) next_chunk<CK>(w, c);
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

template <int D, bool ONE>
int run(const TcParams& p, cudaStream_t s) {
    if (ensure_dynamic_smem(reinterpret_cast<const void*>(&k_key_weights_tc<D, ONE>), Cfg<D>::SMEM)) return -1;
    k_key_weights_tc<D, ONE><<<p.w.a.n_cta, THREADS, Cfg<D>::SMEM, s>>>(p);
    return 0;
}

}  // namespace

bool key_weights_tc_supported(int dtype, const KeyWeightArgs& w) {
    int box = 0;
    const PagedAttnArgs& a = w.a;
    return dtype == 1 && (a.D == 64 || a.D == 128) && a.group <= PAIRS && paged_tma_pages(a, SUB, &box) && reinterpret_cast<uintptr_t>(a.q.p) % 16 == 0 &&
           a.q.tok % 8 == 0 && a.q.head % 8 == 0 && a.q.tok < (1ll << 39) && a.q.head < (1ll << 39) && (a.q.tok > 0 || a.seq.n_tokens == 1) && (a.q.head > 0 || a.Hq == 1);
}

int launch_key_weights_tc(KeyWeightArgs w, int n_sm, cudaStream_t s) {
    TcParams p;
    memset(&p, 0, sizeof(p));
    PagedAttnArgs& a = w.a;
    if (!paged_tma_pages(a, SUB, &p.box_rows) || paged_page_map(&p.map_k, a, a.pages.k, p.box_rows)) return -1;
    a.rows = PAIRS / a.group;
    a.rows_shift = shift_of(a.rows);
    {
        EncodeFn enc = get_encode();
        cuuint64_t dims[3] = {(cuuint64_t)a.D, (cuuint64_t)a.Hq, (cuuint64_t)a.seq.n_tokens};
        cuuint64_t strides[2] = {(cuuint64_t)(a.q.head > 0 ? a.q.head * 2 : a.D * 2), (cuuint64_t)(a.q.tok > 0 ? a.q.tok * 2 : a.D * 2)};
        cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)a.rows};
        const cuuint32_t estr[3] = {1, 1, 1};
        if (enc(&p.map_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, a.q.p, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) return -1;
    }
    p.group_inv = (65536 + a.group - 1) / a.group;
    a.n_cta = n_sm;
    a.min_units = 1;
    p.w = w;
    const long long observed = w.last > 0 && w.last < a.seq.max_new ? w.last : a.seq.max_new;
    // (then no chunk has two owners either)
    if (observed <= a.rows) return a.D == 128 ? run<128, true>(p, s) : run<64, true>(p, s);
    const int rc = a.D == 128 ? run<128, false>(p, s) : run<64, false>(p, s);
    return rc ? rc : launch_key_weights_join(w, CK, s);
}

}  // namespace esp
