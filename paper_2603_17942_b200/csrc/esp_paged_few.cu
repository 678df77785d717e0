// Attention of single tokens over pages: bf16, heads of 64 or 128, one new token per sequence, up to 16 query heads per KV head.
//
// Every cached key and value is read once for a handful of rows, so memory bounds it, and what counts is that every SM always has
// loads under way.  Each warp is a worker of its own, with a share of the line of units, a ring of stages and no partner to wait for:
// its lane 0 requests the pages' slots of a stage by TMA (both halves of a head's elements in one box), the warp takes a stage of KEYS keys
// when it has landed and requests the next one into its place.  The products are m16n8k16: rows the query heads, Q in registers
// for the whole tile, keys and values as ldmatrix gives them.  Weights go as two bf16 numbers, hi + lo (up to 8 heads: hi in rows 0-7 and lo in rows
// 8-15 of one operand), so that they lose nothing against the output's own rounding; the tensor cores have the time.
// The one new token sees the same positions in all rows: what it does not see is cut off the ends, its values are set to zero in registers.
#include <string.h>

#include "esp_attn_tc.cuh"
#include "esp_paged.cuh"

namespace esp {

namespace {

using namespace tc;
using namespace paged;

// Warps and stages of the 192 KB (us, 64 sequences of 1k to 8k positions / 8 of 32k): 3 x 4 of 16 KB 220 / 247, 4 x 3 170 / 191, 6 x 2 147 / 175, 7 x 2 151 / 179;
// of 8 KB 6 x 4 159 / 190, 8 x 3 150 / 188, 12 x 2 150 / 182.  A warp's own chain per stage is what more warps hide.
constexpr int WARPS = 6, STAGES = 2, STAGE_BYTES = 16384;
constexpr int SMEM = 1024 + WARPS * STAGES * STAGE_BYTES + 256;

struct FewParams {
    CUtensorMap map_k;    // [pages][heads][halves][slots][64], box 64 x box_rows x halves
    CUtensorMap map_v;
    PagedAttnArgs a;
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
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t pack(float x, float y) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&b);
}
// hi + lo = the weights x, y to 16 bits.  hi is cut off and lo taken of a weight one fp32 step larger, so that both are positive down to weights of 2^-103: an infinite value times
// hi plus the same times lo is infinite.  (With hi rounded lo was zero or negative for many weights, a single key's 1 among them, and the sum no number.)
__device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo) {
    constexpr float UP = 1.f + 0x1p-23f;
    hi = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
    lo = pack(fmaf(x, UP, -__uint_as_float(hi << 16)), fmaf(y, UP, -__uint_as_float(hi & 0xffff0000u)));
}

// Registers for one block per SM, which is what shared memory allows; heads of 128 are left to the compiler (us, 64 sequences of 1k to 8k, bounded / not: 4 KV heads of 64
// with 64 query heads 55.7 / 59.8, where it spilled for a second block; 8 of 128 with 32 149.7 / 147.9, 8 sequences of 32k 179 / 173).
template <int D, bool G8>
__global__ void __launch_bounds__(WARPS * 32, D == 64 ? 1 : 0) k_paged_few(const __grid_constant__ FewParams p) {
    constexpr int HALVES = D / 64, KEYS = STAGE_BYTES / (D * 4), NT = KEYS / 8, HALF_STAGE = STAGE_BYTES / 2;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned char* ring = smem + warp * STAGES * STAGE_BYTES;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + WARPS * STAGES * STAGE_BYTES) + warp * STAGES;
    volatile int* s_abort = reinterpret_cast<volatile int*>(smem + WARPS * STAGES * STAGE_BYTES + WARPS * STAGES * 8) + warp;
    const PagedAttnArgs& a = p.a;
    const int worker = warp * gridDim.x + blockIdx.x;       // the first workers on SMs of their own
    if (lane == 0) {
        prefetch_tensormap(&p.map_k);
        prefetch_tensormap(&p.map_v);
        for (int i = 0; i < STAGES; ++i) mbar_init(&full[i], 1);
        *s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    pdl_launch_dependents();
    Share share;
    Cursor c;
    Descs desc;
    desc.clear();
    if (!deal<KEYS>(a, worker, lane, share, c)) {
        if (lane == 0) desc.store(a, worker);
        return;
    }
    const uint32_t begin = share.begin(worker), end = share.begin(worker + 1);

    // ---- requests, up to STAGES units ahead of the products
    Cursor ci = c;
    uint32_t ui = begin;
    const int n_boxes = KEYS >> p.box_shift, box_bytes = (128 * HALVES) << p.box_shift;
    int page = 0, slot = 0;
    auto look_up = [&]() {              // the pages of unit ui, a lane per box
        const int pos = (ci.x.c0 + (int)(ui - ci.tile_u)) * KEYS + ((lane & (n_boxes - 1)) << p.box_shift);
        page = a.pages.n_pages;         // a page that there is not reads as zeros
        slot = 0;
        if (pos < ci.s.kv && pos + (1 << p.box_shift) > first_seen(a, ci.s, 0)) {
            const int index = page_index(a.pages, pos);
            const int pg = load_page(a.seq, a.pages, ci.b, index);
            if (pg >= 0) page = pg;
            slot = pos - index * a.pages.page_size;
        }
    };
    auto request = [&]() {
        const uint32_t st = (ui - begin) % STAGES;
        unsigned char* dst = ring + st * STAGE_BYTES;
        if (lane == 0) mbar_expect_tx(&full[st], STAGE_BYTES);
        for (int i = 0; i < n_boxes; ++i) {
            const int pg = __shfl_sync(0xffffffffu, page, i), sl = __shfl_sync(0xffffffffu, slot, i);
            if (lane == 0) {
                tma_load_5d(dst + i * box_bytes, &p.map_k, sl, ci.kvh, pg, &full[st]);
                tma_load_5d(dst + HALF_STAGE + i * box_bytes, &p.map_v, sl, ci.kvh, pg, &full[st]);
            }
        }
        __syncwarp();
        if (++ui < end) {
            if (ui - ci.tile_u >= (uint32_t)ci.x.nc) next_tile<KEYS>(a, ci);
            look_up();
        }
    };
    look_up();
    for (int i = 0; i < STAGES && ui < end; ++i) request();

    // ---- products
    const int g = lane >> 2, c4 = lane & 3;
    // shared-memory offset of this lane's row of ldmatrix in a stage: keys lane % 8 (+ 8 for odd matrices of V)
    auto row_off = [&](int r) { return (uint32_t)((r >> p.box_shift) * box_bytes + (r & ((1 << p.box_shift) - 1)) * 128); };
    auto chunk_off = [&](int ch) { return (uint32_t)(((ch >> 3) << (p.box_shift + 7)) + (((ch & 7) ^ (lane & 7)) << 4)); };
    bool ok = true;
    for (uint32_t u = begin; u < end && ok;) {
        const Piece pc = make_piece(c, begin, u, end);
        const int P = c.s.kv - 1, lo = a.window > 0 ? max(0, P - a.window + 1) : 0;       // the token sees [lo, kv)
        uint32_t qa[D / 16][4];
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.q.p) + out_offset(a.q, c.s.start, c.kvh * a.group) + kk * 16 + c4 * 2;
            qa[kk][0] = qa[kk][1] = qa[kk][2] = qa[kk][3] = 0;
            if (g < a.group) {
                qa[kk][0] = __ldg(reinterpret_cast<const uint32_t*>(q + g * a.q.head));
                qa[kk][2] = __ldg(reinterpret_cast<const uint32_t*>(q + g * a.q.head + 8));
            }
            if (!G8 && g + 8 < a.group) {
                qa[kk][1] = __ldg(reinterpret_cast<const uint32_t*>(q + (g + 8) * a.q.head));
                qa[kk][3] = __ldg(reinterpret_cast<const uint32_t*>(q + (g + 8) * a.q.head + 8));
            }
        }
        constexpr int R = G8 ? 1 : 2;       // rows of a lane: g and g + 8
        float m_run[R], l_run[R], o[D / 8][4];
#pragma unroll
        for (int r = 0; r < R; ++r) { m_run[r] = -INFINITY; l_run[r] = 0.f; }
#pragma unroll
        for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;

        for (int j = 0; j < pc.n; ++j, ++u) {
            const uint32_t st = (u - begin) % STAGES;
            if (!__all_sync(0xffffffffu, mbar_wait(&full[st], ((u - begin) / STAGES) & 1, s_abort))) { ok = false; break; }
            const uint32_t k_addr = smem_u32(ring + st * STAGE_BYTES), v_addr = k_addr + HALF_STAGE;
            const int p0 = (pc.c0 + j) * KEYS;
            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
                const uint32_t row = k_addr + row_off(nt * 8 + (lane & 7));
#pragma unroll
                for (int kk = 0; kk < D / 32; ++kk) {
                    uint32_t b[4];
                    ldsm4(b, row + chunk_off(kk * 4 + (lane >> 3)));
                    attn::mma16816(s[nt], qa[2 * kk][0], qa[2 * kk][1], qa[2 * kk][2], qa[2 * kk][3], b[0], b[1]);
                    attn::mma16816(s[nt], qa[2 * kk + 1][0], qa[2 * kk + 1][1], qa[2 * kk + 1][2], qa[2 * kk + 1][3], b[2], b[3]);
                }
            }
            const bool edge = p0 < lo || p0 + KEYS > c.s.kv;      // the same in every lane
            if (edge) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int pos = p0 + nt * 8 + c4 * 2 + (e & 1);
                        if (pos < lo || pos >= c.s.kv) s[nt][e] = -INFINITY;
                    }
            }
            float m_use[R];
            bool any_move = false;
            float alpha[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float cm = -INFINITY;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) cm = fmaxf(cm, fmaxf(s[nt][2 * r], s[nt][2 * r + 1]));
                cm = fmaxf(cm, __shfl_xor_sync(0xffffffffu, cm, 1));
                cm = fmaxf(cm, __shfl_xor_sync(0xffffffffu, cm, 2));
                cm *= a.scale_log2;
                // the reference of the exponentials follows the maximum when it has grown by more than 2^8
                const bool move = m_run[r] == -INFINITY ? cm != -INFINITY : cm - m_run[r] > 8.f;
                const float m_new = move ? cm : m_run[r];
                m_use[r] = m_new == -INFINITY ? 0.f : m_new;
                alpha[r] = m_run[r] == m_use[r] ? 1.f : exp2f(m_run[r] - m_use[r]);
                m_run[r] = m_new;
                any_move = any_move || move;
            }
            if (j > 0 && __any_sync(0xffffffffu, any_move)) {
#pragma unroll
                for (int n = 0; n < D / 8; ++n) {
                    o[n][0] *= alpha[0]; o[n][1] *= alpha[0];
                    o[n][2] *= alpha[R - 1]; o[n][3] *= alpha[R - 1];
                }
#pragma unroll
                for (int r = 0; r < R; ++r) l_run[r] *= alpha[r];
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    s[nt][2 * r] = attn::ex2_approx(fmaf(s[nt][2 * r], a.scale_log2, -m_use[r]));
                    s[nt][2 * r + 1] = attn::ex2_approx(fmaf(s[nt][2 * r + 1], a.scale_log2, -m_use[r]));
                    l_run[r] += s[nt][2 * r] + s[nt][2 * r + 1];
                }
#pragma unroll
            for (int ks = 0; ks < KEYS / 16; ++ks) {
                uint32_t h0, l0, h2, l2, h1 = 0, l1 = 0, h3 = 0, l3 = 0;
                split(s[2 * ks][0], s[2 * ks][1], h0, l0);
                split(s[2 * ks + 1][0], s[2 * ks + 1][1], h2, l2);
                if (!G8) {
                    split(s[2 * ks][2], s[2 * ks][3], h1, l1);
                    split(s[2 * ks + 1][2], s[2 * ks + 1][3], h3, l3);
                }
                uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;      // values of positions that are not seen may be no numbers
                if (edge) {
                    const int k0 = p0 + ks * 16 + c4 * 2;
                    auto in = [&](int pos) { return pos >= lo && pos < c.s.kv; };
                    keep0 = (in(k0) ? 0xffffu : 0u) | (in(k0 + 1) ? 0xffff0000u : 0u);
                    keep1 = (in(k0 + 8) ? 0xffffu : 0u) | (in(k0 + 9) ? 0xffff0000u : 0u);
                }
                const uint32_t row = v_addr + row_off(ks * 16 + ((lane >> 3) & 1) * 8 + (lane & 7));
#pragma unroll
                for (int db = 0; db < D / 16; ++db) {
                    uint32_t b[4];
                    ldsm4_trans(b, row + chunk_off(db * 2 + (lane >> 4)));
                    b[0] &= keep0; b[1] &= keep1; b[2] &= keep0; b[3] &= keep1;
                    if (G8) {
                        attn::mma16816(o[2 * db], h0, l0, h2, l2, b[0], b[1]);
                        attn::mma16816(o[2 * db + 1], h0, l0, h2, l2, b[2], b[3]);
                    } else {
                        attn::mma16816(o[2 * db], h0, h1, h2, h3, b[0], b[1]);
                        attn::mma16816(o[2 * db + 1], h0, h1, h2, h3, b[2], b[3]);
                        attn::mma16816(o[2 * db], l0, l1, l2, l3, b[0], b[1]);
                        attn::mma16816(o[2 * db + 1], l0, l1, l2, l3, b[2], b[3]);
                    }
                }
            }
            __syncwarp();                   // every lane has read the stage
            if (ui < end) request();
        }
        if (!ok) break;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 1);
            l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 2);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int pair = g + 8 * r;
            if (pair >= a.group) continue;
            const int head = c.kvh * a.group + pair;
            const float inv = l_run[r] == 0.f ? 0.f : 1.f / l_run[r];
            __nv_bfloat16* y = reinterpret_cast<__nv_bfloat16*>(a.out.p) + out_offset(a.out, c.s.start, head) + c4 * 2;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
                const float x0 = G8 ? o[n][0] + o[n][2] : o[n][2 * r], x1 = G8 ? o[n][1] + o[n][3] : o[n][2 * r + 1];
                if (pc.slot < 0) {
                    const uint32_t w = pack(x0 * inv, x1 * inv);
                    if (a.out_vec) *reinterpret_cast<uint32_t*>(y + n * 8) = w;
                    else { y[n * 8] = __ushort_as_bfloat16((unsigned short)w); y[n * 8 + 1] = __ushort_as_bfloat16((unsigned short)(w >> 16)); }
                } else {
                    reinterpret_cast<float2*>(a.part_o + part_quad(a, worker, pc.slot, n * 2 + (c4 >> 1), pair))[c4 & 1] = make_float2(x0, x1);
                }
            }
            if (c4 == 0) {
                if (pc.slot >= 0) a.part_ml[part_row(a, worker, pc.slot, pair)] = make_float2(m_run[r], l_run[r]);
                else if (a.lse) a.lse[(size_t)c.s.start * a.Hq + head] = l_run[r] == 0.f ? -INFINITY : (m_run[r] + log2f(l_run[r])) * 0.6931471805599453f;
            }
        }
        desc.note(a, c, share, pc);
        if (u < end) next_tile<KEYS>(a, c);
    }
    if (lane == 0) desc.store(a, worker);
    if (!ok) {
        if (lane == 0) set_error(a.seq.status, DEV_E_WAIT_TIMEOUT);
        for (int i = 0; i < 64; ++i) __nanosleep(10000);    // let copies in flight land before shared memory goes away
    }
}

// The tile whose first piece worker c has as its last one: a warp for every eighth part, a lane for MERGE_ITEMS / 32 quads of a pair, the warps' sums joined
// in order through shared memory.
constexpr int MERGE_WARPS = 8, MERGE_ITEMS = 128;
template <typename T, int D>
__global__ void __launch_bounds__(MERGE_WARPS * 32) k_paged_merge_few(const __grid_constant__ PagedAttnArgs a) {
    __shared__ float4 s_o[MERGE_WARPS][MERGE_ITEMS];
    __shared__ float s_l[MERGE_WARPS][16], s_m[16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x, pairs = a.pairs;      // a power of two, at most 16
    pdl_wait();
    const int4 dd = __ldcg(reinterpret_cast<const int4*>(a.desc + 2 * c));
    const int n_pairs = dd.y, n = dd.w >> 2, first_slot = dd.w & 1;
    if (n == 0) return;
    auto slot_of = [&](int k) { return 2 * k + (k == 0 ? first_slot : 0); };
    const float2* ml = a.part_ml + part_row(a, c, 0, lane & (pairs - 1));
    // the largest reference of each pair: lanes deal the parts among themselves
    float m = -INFINITY;
    const int step = 32 / pairs;
    for (int k0 = lane / pairs; k0 < n; k0 += 4 * step) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = __ldcg(ml + (size_t)slot_of(min(k0 + e * step, n - 1)) * pairs).x;
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, x[e]);
    }
    for (int o = pairs; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float m_use = m == -INFINITY ? 0.f : m;
    constexpr int NI = MERGE_ITEMS / 32;
    const int quads = D / 4;
    float4 acc[NI];
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    // item: pair fastest, as the partials lie; lane and lane + 32 have the same pair
    const int item0 = blockIdx.y * MERGE_ITEMS + lane;
    for (int k0 = warp; k0 < n; k0 += 2 * MERGE_WARPS) {
        float2 x[2];
        float4 v[2][NI];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int sl = slot_of(min(k0 + e * MERGE_WARPS, n - 1));
            x[e] = __ldcg(ml + (size_t)sl * pairs);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int item = item0 + i * 32;
                v[e][i] = item < quads * pairs ? __ldcg(a.part_o + part_quad(a, c, sl, 0, 0) + item) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (k0 + e * MERGE_WARPS >= n) break;
            const float w = exp2f(x[e].x - m_use);
            l = fmaf(x[e].y, w, l);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                acc[i].x = fmaf(v[e][i].x, w, acc[i].x); acc[i].y = fmaf(v[e][i].y, w, acc[i].y);
                acc[i].z = fmaf(v[e][i].z, w, acc[i].z); acc[i].w = fmaf(v[e][i].w, w, acc[i].w);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) s_o[warp][lane + 32 * i] = acc[i];
    if (lane < pairs) s_l[warp][lane] = l;
    if (warp == 0 && lane < pairs) s_m[lane] = m;
    __syncthreads();
    const int item = blockIdx.y * MERGE_ITEMS + threadIdx.x, pr = item & (pairs - 1), dq = item / pairs;
    if (threadIdx.x >= MERGE_ITEMS || dq >= quads || pr >= n_pairs) return;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    l = 0.f;
#pragma unroll
    for (int w = 0; w < MERGE_WARPS; ++w) {
        const float4 x = s_o[w][threadIdx.x];
        t.x += x.x; t.y += x.y; t.z += x.z; t.w += x.w;
        l += s_l[w][pr];
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int row = pr / a.group, head = dd.z + pr - row * a.group, token = dd.x + row;
    store4<T>(reinterpret_cast<T*>(a.out.p) + out_offset(a.out, token, head) + 4 * dq, make_float4(t.x * inv, t.y * inv, t.z * inv, t.w * inv), a.out_vec);
    if (a.lse && dq == 0) a.lse[(size_t)token * a.Hq + head] = l == 0.f ? -INFINITY : (s_m[pr] + log2f(l)) * 0.6931471805599453f;
}

template <int D>
int run_few(FewParams& p, cudaStream_t s) {
    const void* f = p.a.group <= 8 ? reinterpret_cast<const void*>(&k_paged_few<D, true>) : reinterpret_cast<const void*>(&k_paged_few<D, false>);
    if (ensure_dynamic_smem(f, SMEM)) return -1;
    if (p.a.group <= 8) k_paged_few<D, true><<<p.a.n_cta / WARPS, WARPS * 32, SMEM, s>>>(p);
    else k_paged_few<D, false><<<p.a.n_cta / WARPS, WARPS * 32, SMEM, s>>>(p);
    return 0;
}
template <typename T, int D>
int run_merge_few(const PagedAttnArgs& a, cudaStream_t s) {
    return launch_k(k_paged_merge_few<T, D>, dim3(a.n_cta - 1, (a.pairs * (D / 4) + MERGE_ITEMS - 1) / MERGE_ITEMS), dim3(MERGE_WARPS * 32), 0, s, true, a) != cudaSuccess;
}

}  // namespace

int paged_page_map5(CUtensorMap* map, const PagedAttnArgs& a, const void* base, int box_rows) {
    EncodeFn enc = get_encode();
    if (!enc) return -1;
    auto bytes = [&](long long stride) { return (cuuint64_t)(stride > 0 ? stride * 2 : a.D * 2); };      // (a dimension of one element: any stride)
    cuuint64_t dims[5] = {64, (cuuint64_t)a.pages.page_size, (cuuint64_t)(a.D / 64), (cuuint64_t)a.Hkv, (cuuint64_t)a.pages.n_pages};
    cuuint64_t strides[4] = {bytes(a.pages.tok), 128, bytes(a.pages.head), bytes(a.pages.page)};
    cuuint32_t box[5] = {64, (cuuint32_t)box_rows, (cuuint32_t)(a.D / 64), 1, 1};
    const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? 0 : -1;
}

int launch_paged_merge_few(int dtype, const PagedAttnArgs& a, cudaStream_t s) {
    if (a.n_cta < 2) return 0;
    if (dtype == 0) return a.D == 32 ? run_merge_few<float, 32>(a, s) : (a.D == 64 ? run_merge_few<float, 64>(a, s) : run_merge_few<float, 128>(a, s));
    return a.D == 32 ? run_merge_few<__nv_bfloat16, 32>(a, s) : (a.D == 64 ? run_merge_few<__nv_bfloat16, 64>(a, s) : run_merge_few<__nv_bfloat16, 128>(a, s));
}

bool paged_few_supported(int dtype, const PagedAttnArgs& a) {
    int box = 0;
    // (a lane reads two elements of a query at a time)
    return dtype == 1 && (a.D == 64 || a.D == 128) && a.group <= 16 && a.seq.max_new == 1 && !a.anc && paged_tma_pages(a, STAGE_BYTES / (a.D * 4), &box) &&
           reinterpret_cast<uintptr_t>(a.q.p) % 4 == 0 && a.q.tok % 2 == 0 && a.q.head % 2 == 0;
}

int launch_paged_few(PagedAttnArgs a, int n_sm, cudaStream_t s) {
    FewParams p;
    memset(&p, 0, sizeof(p));
    int box = 0;
    if (!paged_tma_pages(a, STAGE_BYTES / (a.D * 4), &box)) return -1;
    if (paged_page_map5(&p.map_k, a, a.pages.k, box) || paged_page_map5(&p.map_v, a, a.pages.v, box)) return -1;
    p.box_shift = shift_of(box);
    a.rows = 1;
    a.rows_shift = 0;
    a.pairs = 1;
    while (a.pairs < a.group) a.pairs *= 2;
    a.n_cta = n_sm * WARPS;
    // Chunks of a worker at least (us in a graph with 1 / 2 / 4 / 8, 32/8 heads of 128): one sequence of 512 9.7 / 10.6 / 12.8 / 17.5, of 4096 16.4 / 13.1 / 14.1 / 18.4, of 16384
    // 27.4 / 27.5 / 26.8 / 23.2; 4 of 1024 12.4 / 11.3 / 13.6 / 18.3; 16 of 512 16.0 / 15.9 / 13.9 / 18.6.  Fewer parts to join against fewer chunks behind one another.
    a.min_units = 2;
    p.a = a;
    const int rc = a.D == 128 ? run_few<128>(p, s) : run_few<64>(p, s);
    return rc ? rc : launch_paged_merge_few(1, a, s);
}

}  // namespace esp
