// Weights of cached positions from a handful of (token, query head) pairs: bf16, heads of 64 or 128, up to 32 observed pairs of a sequence and KV head; and from any number where
// pages or queries do not lie as the tensor cores' boxes want them.
//
// Every cached key is read once, so memory bounds it, as in the attention of single tokens, and it is built the same way: each warp is a worker
// with a share of the line of chunks, a stage of its own that TMA fills, and no partner to wait for.  The products are m16n8k16 with the
// keys as rows, so that what belongs to a key ends in four lanes of a quad: queries in registers for the whole sequence and head, weights and their sum over the
// columns in registers, two shuffles, one number written for each key.  All tokens count as one tile, so no chunk has several owners and nothing is joined; more than 32 pairs are
// taken 32 at a time, with the queries read anew (from the first-level cache) for every chunk.
// Pages that boxes of eight slots do not fit into (PLAIN) are copied row by row, each lane 16 bytes at a time, to where a box would have put them.
// 64 single tokens over 1k to 8k positions, 32/8 heads of 128: 85 us, 0.90 of the copy rate; one over 4k 5.3 us, of which 3 are the way to the first keys.  Pages of 17, 25 x 4 tokens
// over up to 7109 positions, 16/4 heads of 64: 28 us (on CUDA cores 173).  Which products are weights is a bit of a word that each column makes once: asked product by product, the
// chunks that masks cut took up to twice as long (16 x 8 tokens over 1606 positions, 32/8 heads of 128: 40 us, now 28).
#include <string.h>

#include "esp_attn_tc.cuh"
#include "esp_key_weights.cuh"

namespace esp {

namespace {

using namespace tc;
using namespace paged;

// Warps, stages of a warp and their KB (us, 64 sequences of 1k to 8k positions, 32/8 heads of 128): 4 x 3 x 16 178, 6 x 2 x 16 135, 8 x 3 x 8 133, 12 x 2 x 8 104, 10 x 1 x 16 99,
// 16 x 1 x 8 93, 12 x 1 x 16 90, 20 x 1 x 8 and 24 x 1 x 8 88; one sequence of 4k 6.3 with 16 KB, 5.7 with 8.  A warp's own chain through a stage is long beside
// the stage's bytes, so many warps with one stage each do better than few that run ahead.  With more columns the queries' registers leave room for 12.
constexpr int STAGE_BYTES = 8192;
template <int NB> constexpr int WARPS = NB <= 2 ? 20 : 12;
template <int NB> constexpr int SMEM = 1024 + WARPS<NB> * STAGE_BYTES + 512;

struct FewParams {
    CUtensorMap map_k;    // [pages][heads][halves][slots][64], box 64 x box_rows x halves
    KeyWeightArgs w;
    int32_t box_shift;    // log2 of the slots of a box
};

__device__ __forceinline__ void tma_load_5d(void* dst, const CUtensorMap* map, int y, int w, int v, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %3, %5, %6}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(0), "r"(y), "r"(w), "r"(v)
        : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}

// NB: columns of the products in eights; of 4 there may be several passes.
template <int D, int NB, bool PLAIN>
__global__ void __launch_bounds__(WARPS<NB> * 32, 1) k_key_weights_few(const __grid_constant__ FewParams p) {
    constexpr int HALVES = D / 64, KEYS = STAGE_BYTES / (D * 2), MT = KEYS / 16, MINE = (MT + 3) / 4;      // a lane writes the keys of every fourth row of products
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned char* stage = smem + warp * STAGE_BYTES;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + WARPS<NB> * STAGE_BYTES) + warp;
    volatile int* s_abort = reinterpret_cast<volatile int*>(smem + WARPS<NB> * STAGE_BYTES + WARPS<NB> * 8) + warp;
    const KeyWeightArgs& w = p.w;
    const PagedAttnArgs& a = w.a;
    const int worker = warp * gridDim.x + blockIdx.x;       // the first workers on SMs of their own
    if (!PLAIN && lane == 0) {
        prefetch_tensormap(&p.map_k);
        mbar_init(full, 1);
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    pdl_launch_dependents();
    Share share;
    WCursor c;
    if (!deal_keys<KEYS>(w, worker, lane, share, c)) return;
    const uint32_t begin = share.begin(worker), end = share.begin(worker + 1);

    // ---- requests, one unit ahead of the products
    WCursor ci = c;
    uint32_t ui = begin;
    const int n_boxes = KEYS >> p.box_shift, box_bytes = (128 * HALVES) << p.box_shift;
    int page = 0, slot = 0;
    long long at[KEYS / 32];            // PLAIN: where the lane's rows of the unit are, -1: nowhere
    auto look_up = [&]() {              // the pages of unit ui, a lane per box or for every 32nd row
        if (PLAIN) {
            int e[KEYS / 32];
#pragma unroll
            for (int j = 0; j < KEYS / 32; ++j) e[j] = score_entry(w, ci, min(ci.c * KEYS + j * 32 + lane, ci.x.s.kv - 1));
#pragma unroll
            for (int j = 0; j < KEYS / 32; ++j) {
                const int pos = ci.c * KEYS + j * 32 + lane;         // (a page that there is not is recorded where the score's place is looked up)
                at[j] = -1;
                if (pos < ci.x.s.kv && pos >= first_observed(w, ci.x) && e[j] >= 0 && e[j] < a.pages.n_pages)
                    at[j] = e[j] * a.pages.page + (pos - page_index(a.pages, pos) * a.pages.page_size) * a.pages.tok + ci.kvh * a.pages.head;
            }
            return;
        }
        const int pos = ci.c * KEYS + ((lane & (n_boxes - 1)) << p.box_shift);
        page = a.pages.n_pages;         // a page that there is not reads as zeros
        slot = 0;
        if (pos < ci.x.s.kv && pos + (1 << p.box_shift) > first_observed(w, ci.x)) {
            const int index = page_index(a.pages, pos);
            const int pg = load_page(a.seq, a.pages, ci.b, index);
            if (pg >= 0) page = pg;
            slot = pos - index * a.pages.page_size;
        }
    };
    auto request = [&]() {
        if (PLAIN) {
            constexpr int PARTS = D / 8;        // 16 bytes each, of a row
#pragma unroll
            for (int i = 0; i < KEYS * PARTS / 32; ++i) {
                const int r = (i * 32 + lane) / PARTS, ch = lane % PARTS;
                const long long from = __shfl_sync(0xffffffffu, at[i * 32 / PARTS / 32], r & 31);
                copy16(smem_u32(stage) + ((ch >> 3) * KEYS + r) * 128 + (((ch & 7) ^ (r & 7)) << 4), reinterpret_cast<const __nv_bfloat16*>(a.pages.k) + (from < 0 ? 0 : from + ch * 8),
                       from >= 0);
            }
        } else {
            if (lane == 0) mbar_expect_tx(full, STAGE_BYTES);
            for (int i = 0; i < n_boxes; ++i) {
                const int pg = __shfl_sync(0xffffffffu, page, i), sl = __shfl_sync(0xffffffffu, slot, i);
                if (lane == 0) tma_load_5d(stage + i * box_bytes, &p.map_k, sl, ci.kvh, pg, full);
            }
        }
        __syncwarp();
        if (++ui < end) {
            next_chunk<KEYS>(w, ci);
            look_up();
        }
    };
    look_up();
    request();

    // ---- products
    const int g = lane >> 2, c4 = lane & 3;
    auto row_off = [&](int r) { return (uint32_t)((r >> p.box_shift) * box_bytes + (r & ((1 << p.box_shift) - 1)) * 128); };
    auto chunk_off = [&](int ch) { return (uint32_t)(((ch >> 3) << (p.box_shift + 7)) + (((ch & 7) ^ (lane & 7)) << 4)); };
    int entry[MINE][2];                  // the page table's for the positions whose scores this lane writes
    auto entries = [&](const WCursor& k) {
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) entry[m][r] = score_entry(w, k, min(k.c * KEYS + (m * 4 + c4) * 16 + r * 8 + g, k.x.s.kv - 1));
    };
    entries(c);
    bool ok = true;
    int b_of = -1, h_of = -1;            // whose queries the registers hold
    uint32_t qb[D / 16][NB][2];
    float minus[NB][2];                  // -lse in the log2 domain
    uint32_t valid = 0;
    // the pairs of a pass: their queries and lse, for tokens row0 on, the first of them with the head rem0 of its group
    auto take_pairs = [&](const Seq& s, int row0, int rem0, int pairs) {
        valid = 0;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int pr = nb * 8 + g, row = (rem0 + pr) / a.group;
            const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q.p) + out_offset(a.q, s.start + row0 + row, c.kvh * a.group + rem0 + pr - row * a.group) + c4 * 2;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                qb[kk][nb][0] = qb[kk][nb][1] = 0;
                if (pr < pairs) {
                    qb[kk][nb][0] = __ldg(reinterpret_cast<const uint32_t*>(q + kk * 16));
                    qb[kk][nb][1] = __ldg(reinterpret_cast<const uint32_t*>(q + kk * 16 + 8));
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int col = nb * 8 + c4 * 2 + e, r = (rem0 + col) / a.group;
                minus[nb][e] = 0.f;
                if (col < pairs) {
                    minus[nb][e] = __ldg(w.lse + (size_t)(s.start + row0 + r) * a.Hq + c.kvh * a.group + rem0 + col - r * a.group) * -1.4426950408889634f;
                    valid |= 1u << (2 * nb + e);
                }
            }
        }
    };
    for (uint32_t u = begin; u < end; ++u) {
        const Seq& s = c.x.s;
        const int L = s.kv - s.n, p0 = c.c * KEYS;
        const long long pairs = (long long)(s.n - c.x.i0) * a.group;
        const bool once = NB < 4 || !PLAIN || pairs <= NB * 8;      // the queries stay
        if (once && (c.b != b_of || c.kvh != h_of)) {
            b_of = c.b;
            h_of = c.kvh;
            take_pairs(s, c.x.i0, 0, (int)pairs);
        }
        // the places of this lane's scores, and what they hold, while the keys are on their way; the next chunk's table entries for its turn
        float *to[MINE][2], old[MINE][2];
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int pos = p0 + (m * 4 + c4) * 16 + r * 8 + g;
                to[m][r] = pos < s.kv && m * 4 + c4 < MT ? score_of(w, c, pos, entry[m][r]) : nullptr;
                old[m][r] = 0.f;
                if (to[m][r] && has_old(w, s, pos)) old[m][r] = *to[m][r];
            }
        WCursor cn = c;
        if (u + 1 < end) next_chunk<KEYS>(w, cn);
        entries(cn);
        if (PLAIN) {
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
        } else if (!__all_sync(0xffffffffu, mbar_wait(full, (u - begin) & 1, s_abort))) { ok = false; break; }
        const uint32_t k_addr = smem_u32(stage);
        float sum[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sum[mt][0] = sum[mt][1] = 0.f;
        for (long long done = 0; done == 0 || (!once && done < pairs); done += NB * 8) {
            const int row0 = c.x.i0 + (int)(once ? 0 : done / a.group), rem0 = once ? 0 : (int)(done % a.group), here = (int)min((long long)(once ? pairs : NB * 8), pairs - done);
            const int row1 = once ? s.n - 1 : row0 + (rem0 + here - 1) / a.group;
            if (!once) {
                if (!a.anc && (p0 > L + row1 || (a.window > 0 && p0 + KEYS <= L + row0 - a.window + 1))) continue;       // nobody sees any of it
                take_pairs(s, row0, rem0, here);
            }
            // a chunk that some token does not see as a whole
            const bool edge = p0 + KEYS > (a.anc ? L : L + row0 + 1) || (a.window > 0 && p0 < L + row1 + 1 - a.window);
            // which of the lane's products are weights, a bit each: column by column its keys
            constexpr int PER = MT * 2, WORDS = (NB * 2 * PER + 31) / 32;
            uint32_t vis[WORDS];
#pragma unroll
            for (int i = 0; i < WORDS; ++i) vis[i] = 0;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t bits = (valid >> (2 * nb + e)) & 1 ? (1u << PER) - 1u : 0u;
                    if (edge && bits) {
                        const RowMask m = row_mask(a, s, row0 + (rem0 + nb * 8 + c4 * 2 + e) / a.group);
                        bits = 0;
#pragma unroll
                        for (int k = 0; k < PER; ++k) bits |= (uint32_t)sees(m, p0 + k * 8 + g, L, s.kv) << k;
                    }
                    vis[(2 * nb + e) * PER / 32] |= bits << ((2 * nb + e) * PER % 32);
                }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float x[NB][4];
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) x[nb][0] = x[nb][1] = x[nb][2] = x[nb][3] = 0.f;
                const uint32_t row = k_addr + row_off(mt * 16 + (lane & 15));
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    uint32_t k[4];
                    ldsm4(k, row + chunk_off(kk * 2 + (lane >> 4)));
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) attn::mma16816(x[nb], k[0], k[1], k[2], k[3], qb[kk][nb][0], qb[kk][nb][1]);
                }
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int bit = (2 * nb + (e & 1)) * PER + mt * 2 + (e >> 1);
                        const bool in = (vis[bit / 32] >> (bit % 32)) & 1;
                        const float y = attn::ex2_approx(fmaf(x[nb][e], a.scale_log2, minus[nb][e & 1]));
                        sum[mt][e >> 1] += in ? y : 0.f;
                    }
            }
        }
        __syncwarp();                   // every lane has read the stage
        if (ui < end) request();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                sum[mt][r] += __shfl_xor_sync(0xffffffffu, sum[mt][r], 1);
                sum[mt][r] += __shfl_xor_sync(0xffffffffu, sum[mt][r], 2);
            }
#pragma unroll
        for (int m = 0; m < MINE; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float x = sum[m * 4][r];
#pragma unroll
                for (int q = 1; q < 4 && m * 4 + q < MT; ++q) x = c4 == q ? sum[m * 4 + q][r] : x;
                if (to[m][r]) *to[m][r] = fmaf(w.keep, old[m][r], x);
            }
        c = cn;
    }
    if (!ok) {
        if (lane == 0) set_error(a.seq.status, DEV_E_WAIT_TIMEOUT);
        for (int i = 0; i < 64; ++i) __nanosleep(10000);    // let copies in flight land before shared memory goes away
    }
}

int observed_pairs(const KeyWeightArgs& w) {
    const long long tokens = w.last > 0 && w.last < w.a.seq.max_new ? w.last : w.a.seq.max_new, pairs = tokens * w.a.group;
    return pairs > 1024 ? 1024 : (int)pairs;
}

template <int D, int NB, bool PLAIN>
int run(FewParams& p, int n_sm, cudaStream_t s) {
    if (ensure_dynamic_smem(reinterpret_cast<const void*>(&k_key_weights_few<D, NB, PLAIN>), SMEM<NB>)) return -1;
    p.w.a.n_cta = n_sm * WARPS<NB>;
    k_key_weights_few<D, NB, PLAIN><<<n_sm, WARPS<NB> * 32, SMEM<NB>, s>>>(p);
    return 0;
}
template <int D, bool PLAIN>
int run(FewParams& p, int n_sm, cudaStream_t s) {
    const int pairs = observed_pairs(p.w);
    return pairs <= 8 ? run<D, 1, PLAIN>(p, n_sm, s) : (pairs <= 16 ? run<D, 2, PLAIN>(p, n_sm, s) : run<D, 4, PLAIN>(p, n_sm, s));
}

}  // namespace

bool key_weights_few_supported(int dtype, const KeyWeightArgs& w) { return observed_pairs(w) <= 32 && key_weights_rows_supported(dtype, w); }
bool key_weights_rows_supported(int dtype, const KeyWeightArgs& w) {
    const PagedAttnArgs& a = w.a;
    // (a lane reads two elements of a query at a time, and copies eight of a key)
    return dtype == 1 && (a.D == 64 || a.D == 128) && reinterpret_cast<uintptr_t>(a.q.p) % 4 == 0 && a.q.tok % 2 == 0 && a.q.head % 2 == 0 &&
           reinterpret_cast<uintptr_t>(a.pages.k) % 16 == 0 && a.pages.page % 8 == 0 && a.pages.tok % 8 == 0 && a.pages.head % 8 == 0;
}

int launch_key_weights_few(KeyWeightArgs w, int n_sm, cudaStream_t s) {
    FewParams p;
    memset(&p, 0, sizeof(p));
    PagedAttnArgs& a = w.a;
    int box = 0;
    const int keys = STAGE_BYTES / (a.D * 2);
    const bool plain = observed_pairs(w) > 32 || !paged_tma_pages(a, keys, &box);
    if (plain) box = keys;
    else if (paged_page_map5(&p.map_k, a, a.pages.k, box)) return -1;
    p.box_shift = shift_of(box);
    a.rows = one_tile(w);
    a.rows_shift = shift_of(a.rows);
    a.min_units = 1;
    p.w = w;
    if (plain) return a.D == 128 ? run<128, true>(p, n_sm, s) : run<64, true>(p, n_sm, s);
    return a.D == 128 ? run<128, false>(p, n_sm, s) : run<64, false>(p, n_sm, s);
}

}  // namespace esp
