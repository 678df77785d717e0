// Attention over pages on CUDA cores (fp32, and bf16 where the tensor-core kernels do not take the head size, page size or alignment),
// and the kernel that joins the split partials of all of them.
//
// A block takes tiles of MP (token, head) pairs that share a KV head and walks their keys 64 at a time: keys and values of a chunk
// in shared memory as fp32, scores, running maximum and sum, P through shared memory, O in registers.  Thread (ty, tx), 16 x 16: pairs
// ty * MP/16 .., keys tx + 16 j of the scores, dims 4 tx + 64 j of the output.
#include "esp_paged.cuh"

namespace esp {

namespace {

using namespace paged;

constexpr int CK = 64;                // keys per chunk
constexpr int THREADS = 256;

template <int D, int MP>
struct SimtSmem {
    float q[MP][D + 4];
    float k[CK][D + 4];
    float v[CK][D];
    float p[MP][CK + 4];
    long long base[CK];               // element offset of the chunk's keys in the pages, -1: none
};

template <typename T, bool VEC>
__device__ __forceinline__ float4 load4(const T* x) {
    if constexpr (!VEC) return make_float4(to_f32(x[0]), to_f32(x[1]), to_f32(x[2]), to_f32(x[3]));
    else if constexpr (sizeof(T) == 4) return __ldg(reinterpret_cast<const float4*>(x));
    else {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(x));
        return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
    }
}
__device__ __forceinline__ bool finite4(const float4& x) { return isfinite(x.x) && isfinite(x.y) && isfinite(x.z) && isfinite(x.w); }

template <typename T, int D, int MP, bool VEC>
__global__ void __launch_bounds__(THREADS) k_paged_simt(const __grid_constant__ PagedAttnArgs a) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SimtSmem<D, MP>& sm = *reinterpret_cast<SimtSmem<D, MP>*>(smem_raw);
    constexpr int PR = MP / 16;                       // pairs of a thread
    constexpr int DV = D >= 64 ? D / 64 : 1;          // float4 columns of a thread (D = 32: the first eight tx have one)
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    pdl_launch_dependents();
    Share share;
    Cursor c;
    Descs desc;
    desc.clear();
    if (!deal<CK>(a, blockIdx.x, tid & 31, share, c)) {
        if (tid == 0) desc.store(a, blockIdx.x);
        return;
    }
    const uint32_t begin = share.begin(blockIdx.x), end = share.begin(blockIdx.x + 1);
    const bool dims = D >= 64 || tx < 8;

    for (uint32_t u = begin; u < end;) {
        const Piece pc = make_piece(c, begin, u, end);
        const int L = c.s.kv - c.s.n, n_pairs = c.x.nr * a.group;
        __syncthreads();                              // the previous piece is done with shared memory
        for (int i = tid; i < MP * (D / 4); i += THREADS) {
            const int pr = i / (D / 4), d = (i % (D / 4)) * 4;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (pr < n_pairs) {
                const int row = pr / a.group, head = c.kvh * a.group + pr - row * a.group;
                x = load4<T, VEC>(reinterpret_cast<const T*>(a.q.p) + out_offset(a.q, c.s.start + c.x.r0 + row, head) + d);
            }
            *reinterpret_cast<float4*>(&sm.q[pr][d]) = x;
        }
        RowMask mask[PR];
        float m_run[PR], l_run[PR];
        float4 o[PR][DV];
#pragma unroll
        for (int i = 0; i < PR; ++i) {
            const int pr = ty * PR + i;
            mask[i].lo = mask[i].hi = 0;
            mask[i].b0 = mask[i].b1 = 0;
            if (pr < n_pairs) mask[i] = row_mask(a, c.s, c.x.r0 + pr / a.group);
            m_run[i] = -INFINITY;
            l_run[i] = 0.f;
#pragma unroll
            for (int j = 0; j < DV; ++j) o[i][j] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        for (int ch = 0; ch < pc.n; ++ch) {
            const int p0 = (pc.c0 + ch) * CK;
            __syncthreads();                          // the previous chunk is done with K, V and P
            if (tid < CK) {
                const int pos = p0 + tid;
                long long base = -1;
                if (pos < c.s.kv && pos >= first_seen(a, c.s, c.x.r0)) {
                    const int index = page_index(a.pages, pos);
                    const int page = load_page(a.seq, a.pages, c.b, index);
                    if (page >= 0) base = page * a.pages.page + (pos - index * a.pages.page_size) * a.pages.tok + c.kvh * a.pages.head;
                }
                sm.base[tid] = base;
            }
            __syncthreads();
            bool odd = false;                         // a value that is infinite or no number
            for (int i = tid; i < CK * (D / 4); i += THREADS) {
                const int r = i / (D / 4), d = (i % (D / 4)) * 4;
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
                if (sm.base[r] >= 0) {
                    x = load4<T, VEC>(reinterpret_cast<const T*>(a.pages.k) + sm.base[r] + d);
                    y = load4<T, VEC>(reinterpret_cast<const T*>(a.pages.v) + sm.base[r] + d);
                    odd = odd || !finite4(y);
                }
                *reinterpret_cast<float4*>(&sm.k[r][d]) = x;
                *reinterpret_cast<float4*>(&sm.v[r][d]) = y;
            }
            odd = __syncthreads_or(odd);
            float s[PR][4];
#pragma unroll
            for (int i = 0; i < PR; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                float4 qv[PR], kv[4];
#pragma unroll
                for (int i = 0; i < PR; ++i) qv[i] = *reinterpret_cast<const float4*>(&sm.q[ty * PR + i][d]);
#pragma unroll
                for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][d]);
#pragma unroll
                for (int i = 0; i < PR; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        s[i][j] = fmaf(qv[i].x, kv[j].x, fmaf(qv[i].y, kv[j].y, fmaf(qv[i].z, kv[j].z, fmaf(qv[i].w, kv[j].w, s[i][j]))));
            }
#pragma unroll
            for (int i = 0; i < PR; ++i) {
                bool vis[4];
                float cm = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    vis[j] = sees(mask[i], p0 + tx + 16 * j, L, c.s.kv);
                    s[i][j] *= a.scale_log2;
                    if (vis[j]) cm = fmaxf(cm, s[i][j]);
                }
#pragma unroll
                for (int w = 8; w > 0; w >>= 1) cm = fmaxf(cm, __shfl_xor_sync(0xffffffffu, cm, w));
                const float m_new = fmaxf(m_run[i], cm), m_use = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = exp2f(m_run[i] - m_use);
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = vis[j] ? exp2f(s[i][j] - m_use) : 0.f;
                    sum += e;
                    // in a chunk with values that are no finite numbers a key that is not seen is told from one of weight 0 by its sign
                    sm.p[ty * PR + i][tx + 16 * j] = odd && !vis[j] ? -1.f : e;
                }
#pragma unroll
                for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
                l_run[i] = fmaf(l_run[i], alpha, sum);
                m_run[i] = m_new;
#pragma unroll
                for (int j = 0; j < DV; ++j) { o[i][j].x *= alpha; o[i][j].y *= alpha; o[i][j].z *= alpha; o[i][j].w *= alpha; }
            }
            __syncthreads();
            if (!odd) {
#pragma unroll 2
                for (int kk = 0; kk < CK; kk += 4) {
                    float4 pv[PR];
#pragma unroll
                    for (int i = 0; i < PR; ++i) pv[i] = *reinterpret_cast<const float4*>(&sm.p[ty * PR + i][kk]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int j = 0; j < DV; ++j) {
                            const float4 vv = *reinterpret_cast<const float4*>(&sm.v[kk + e][dims ? tx * 4 + 64 * j : 0]);
#pragma unroll
                            for (int i = 0; i < PR; ++i) {
                                const float w = e == 0 ? pv[i].x : (e == 1 ? pv[i].y : (e == 2 ? pv[i].z : pv[i].w));
                                o[i][j].x = fmaf(w, vv.x, o[i][j].x); o[i][j].y = fmaf(w, vv.y, o[i][j].y);
                                o[i][j].z = fmaf(w, vv.z, o[i][j].z); o[i][j].w = fmaf(w, vv.w, o[i][j].w);
                            }
                        }
                }
            } else {
                for (int kk = 0; kk < CK; ++kk)
#pragma unroll
                    for (int i = 0; i < PR; ++i) {
                        const float w = sm.p[ty * PR + i][kk];
                        if (w < 0.f) continue;
#pragma unroll
                        for (int j = 0; j < DV; ++j) {
                            const float4 vv = *reinterpret_cast<const float4*>(&sm.v[kk][dims ? tx * 4 + 64 * j : 0]);
                            o[i][j].x = fmaf(w, vv.x, o[i][j].x); o[i][j].y = fmaf(w, vv.y, o[i][j].y);
                            o[i][j].z = fmaf(w, vv.z, o[i][j].z); o[i][j].w = fmaf(w, vv.w, o[i][j].w);
                        }
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < PR; ++i) {
            const int pr = ty * PR + i;
            if (pr >= n_pairs) continue;
            if (pc.slot < 0) {
                const int row = pr / a.group, head = c.kvh * a.group + pr - row * a.group, token = c.s.start + c.x.r0 + row;
                const float inv = l_run[i] == 0.f ? 0.f : 1.f / l_run[i];
                T* y = reinterpret_cast<T*>(a.out.p) + out_offset(a.out, token, head);
                if (dims)
#pragma unroll
                    for (int j = 0; j < DV; ++j)
                        store4<T>(y + tx * 4 + 64 * j, make_float4(o[i][j].x * inv, o[i][j].y * inv, o[i][j].z * inv, o[i][j].w * inv), a.out_vec);
                if (a.lse && tx == 0) a.lse[(size_t)token * a.Hq + head] = l_run[i] == 0.f ? -INFINITY : (m_run[i] + log2f(l_run[i])) * 0.6931471805599453f;
            } else {
                if (dims)
#pragma unroll
                    for (int j = 0; j < DV; ++j) a.part_o[part_quad(a, blockIdx.x, pc.slot, tx + 16 * j, pr)] = o[i][j];
                if (tx == 0) a.part_ml[part_row(a, blockIdx.x, pc.slot, pr)] = make_float2(m_run[i], l_run[i]);
            }
        }
        desc.note(a, c, share, pc);
        u += pc.n;
        if (u < end) next_tile<CK>(a, c);
    }
    if (tid == 0) desc.store(a, blockIdx.x);
}

// Joins the split partials: column x of blocks takes its share of the tiles that CTA x has pieces of, every CTA's column the same
// amount, however many parts a tile has.  A task is 32 pairs x 4 quads (a lane has a pair, as the partials lie); its parts are dealt to 1, 2, 4 or 8 warps, each of
// which weighs its own by 2^(m - its maximum), and the warps' sums are joined in order through shared memory.  (One warp for all
// parts and all tasks of a tile in the column of its first CTA: a call with 18 parts per tile, 32 tokens over 4k positions, took 31 us
// instead of 22.)
constexpr int MERGE_WARPS = 8, MERGE_QUADS = 4, MERGE_PARTS = 4, MERGE_SECOND = PAGED_MAX_PAIRS / 2, MERGE_BLOCKS = 8;

template <typename T, int D>
__global__ void __launch_bounds__(MERGE_WARPS * 32) k_paged_merge(const __grid_constant__ PagedAttnArgs a) {
    __shared__ float4 s_o[MERGE_WARPS][MERGE_QUADS][32];
    __shared__ float2 s_ml[MERGE_WARPS][32];
    constexpr int COLS = D / 4 / MERGE_QUADS;                                   // tasks for the quads of a pair
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, x = blockIdx.x;
    pdl_wait();
    // half of the column's blocks for the tile that starts in CTA x, half for the one that goes on in it
    const int4* dp = reinterpret_cast<const int4*>(a.desc + 2 * x + (blockIdx.y & 1));
    const int4 dd = __ldcg(dp);
    const int c = __ldcg(dp + 1).x, token = dd.x, n_pairs = dd.y, head0 = dd.z, code = dd.w;
    {
        if (code == 0) return;
        const int ctas = code >> 2, two = code >> 1 & 1, n = ctas << two, first_slot = code & 1;
        const int wp = n <= 4 ? 1 : (n <= 8 ? 2 : (n <= 16 ? 4 : 8)), w = warp & (wp - 1);      // warps of a task
        const int tasks = (n_pairs + 31) / 32 * COLS;
        // tasks x - c, x - c + ctas, .. are this column's; its blocks take them in turn, MERGE_WARPS / wp at a time
        for (int m0 = (blockIdx.y >> 1) * (MERGE_WARPS / wp); x - c + m0 * ctas < tasks; m0 += MERGE_BLOCKS / 2 * (MERGE_WARPS / wp)) {
            const int task = x - c + (m0 + warp / wp) * ctas;
            const int pr = task / COLS * 32 + lane, q0 = task % COLS * MERGE_QUADS;
            const bool valid = task < tasks && pr < n_pairs;
            float m = -INFINITY, l = 0.f;
            float4 o[MERGE_QUADS];
#pragma unroll
            for (int i = 0; i < MERGE_QUADS; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (valid) {
                // (two parts of a CTA, where two groups of warps took its chunks in turn: the second one's pairs behind the first one's)
                for (int k0 = w; k0 < n; k0 += wp * MERGE_PARTS) {
                    float2 ml[MERGE_PARTS];
                    float4 v[MERGE_PARTS][MERGE_QUADS];
#pragma unroll
                    for (int e = 0; e < MERGE_PARTS; ++e) {
                        const int k = min(k0 + e * wp, n - 1), cta = k >> two, slot = cta == 0 ? first_slot : 0, at = pr + (two && (k & 1) ? MERGE_SECOND : 0);
                        ml[e] = __ldcg(a.part_ml + part_row(a, c + cta, slot, at));
#pragma unroll
                        for (int i = 0; i < MERGE_QUADS; ++i) v[e][i] = __ldcg(a.part_o + part_quad(a, c + cta, slot, q0 + i, at));
                    }
#pragma unroll
                    for (int e = 0; e < MERGE_PARTS; ++e) {
                        if (k0 + e * wp >= n || ml[e].y == 0.f) continue;      // (a part that saw nothing may have left its values as they were)
                        const float m_new = fmaxf(m, ml[e].x), old = m == m_new ? 1.f : exp2f(m - m_new), wt = ml[e].x == m_new ? 1.f : exp2f(ml[e].x - m_new);
                        l = fmaf(ml[e].y, wt, l * old);
#pragma unroll
                        for (int i = 0; i < MERGE_QUADS; ++i) {
                            o[i].x = fmaf(v[e][i].x, wt, o[i].x * old); o[i].y = fmaf(v[e][i].y, wt, o[i].y * old);
                            o[i].z = fmaf(v[e][i].z, wt, o[i].z * old); o[i].w = fmaf(v[e][i].w, wt, o[i].w * old);
                        }
                        m = m_new;
                    }
                }
            }
            if (wp > 1) {
                s_ml[warp][lane] = make_float2(m, l);
#pragma unroll
                for (int i = 0; i < MERGE_QUADS; ++i) s_o[warp][i][lane] = o[i];
                __syncthreads();
                const int w0 = warp - w;                                        // the task's first warp
                m = -INFINITY;
                for (int k = 0; k < wp; ++k) m = fmaxf(m, s_ml[w0 + k][lane].x);
                l = 0.f;
#pragma unroll
                for (int i = 0; i < MERGE_QUADS; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int k = 0; k < wp; ++k) {
                    const float2 ml = s_ml[w0 + k][lane];
                    if (ml.y == 0.f) continue;
                    const float wt = ml.x == m ? 1.f : exp2f(ml.x - m);
                    l = fmaf(ml.y, wt, l);
#pragma unroll
                    for (int i = 0; i < MERGE_QUADS; ++i) {
                        if (i % wp != w) continue;                              // a quad for each of the warps
                        const float4 y = s_o[w0 + k][i][lane];
                        o[i].x = fmaf(y.x, wt, o[i].x); o[i].y = fmaf(y.y, wt, o[i].y); o[i].z = fmaf(y.z, wt, o[i].z); o[i].w = fmaf(y.w, wt, o[i].w);
                    }
                }
            }
            if (valid) {
                const int row = pr / a.group, head = head0 + pr - row * a.group;
                const float inv = l == 0.f ? 0.f : 1.f / l;
                T* y = reinterpret_cast<T*>(a.out.p) + out_offset(a.out, token + row, head);
#pragma unroll
                for (int i = 0; i < MERGE_QUADS; ++i)
                    if (wp == 1 || i % wp == w) store4<T>(y + 4 * (q0 + i), make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv), a.out_vec);
                if (a.lse && q0 == 0 && w == 0) a.lse[(size_t)(token + row) * a.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            }
            if (wp > 1) __syncthreads();                                        // shared memory is free for the next round
        }
    }
}

template <typename T, int D, int MP, bool VEC>
int run_simt(const PagedAttnArgs& a, cudaStream_t s) {
    const int bytes = (int)sizeof(SimtSmem<D, MP>);
    if (ensure_dynamic_smem(reinterpret_cast<const void*>(&k_paged_simt<T, D, MP, VEC>), bytes)) return -1;
    k_paged_simt<T, D, MP, VEC><<<a.n_cta, THREADS, bytes, s>>>(a);
    return 0;
}
template <typename T, int D>
int run_simt_d(const PagedAttnArgs& a, cudaStream_t s) {
    if (a.pairs == 16) return a.vec ? run_simt<T, D, 16, true>(a, s) : run_simt<T, D, 16, false>(a, s);
    return a.vec ? run_simt<T, D, 64, true>(a, s) : run_simt<T, D, 64, false>(a, s);
}
template <typename T>
int run_simt_t(const PagedAttnArgs& a, cudaStream_t s) {
    return a.D == 32 ? run_simt_d<T, 32>(a, s) : (a.D == 64 ? run_simt_d<T, 64>(a, s) : run_simt_d<T, 128>(a, s));
}

template <typename T, int D>
int run_merge(const PagedAttnArgs& a, cudaStream_t s) {
    return launch_k(k_paged_merge<T, D>, dim3(a.n_cta, MERGE_BLOCKS), dim3(MERGE_WARPS * 32), 0, s, true, a) != cudaSuccess;
}

}  // namespace

int launch_paged_merge(int dtype, const PagedAttnArgs& a, cudaStream_t s) {
    if (dtype == 0) return a.D == 32 ? run_merge<float, 32>(a, s) : (a.D == 64 ? run_merge<float, 64>(a, s) : run_merge<float, 128>(a, s));
    return a.D == 32 ? run_merge<__nv_bfloat16, 32>(a, s) : (a.D == 64 ? run_merge<__nv_bfloat16, 64>(a, s) : run_merge<__nv_bfloat16, 128>(a, s));
}

int launch_paged_simt(int dtype, PagedAttnArgs a, int n_sm, cudaStream_t s) {
    // Small tiles in small calls: more blocks at once, at a higher price per pair.  696 pairs in all (5 sequences of up to 100 tokens, heads of 64)
    // 25.5 us with tiles of 64 pairs, 18.6 with 16; 3200 pairs (4 of up to 300) 43 and 54.
    const bool few = (long long)a.group * a.seq.max_new <= 16 || (long long)a.seq.n_tokens * a.Hq < 16ll * n_sm;
    a.pairs = few && a.group <= 16 ? 16 : 64;
    a.rows = a.pairs / a.group;
    if (a.rows < 1) return -1;                      // more than 64 query heads share a KV head
    a.rows_shift = shift_of(a.rows);
    a.n_cta = n_sm * (a.pairs == 16 ? 4 : 2);
    a.min_units = 1;
    const int rc = dtype == 0 ? run_simt_t<float>(a, s) : run_simt_t<__nv_bfloat16>(a, s);
    if (rc) return rc;
    return a.pairs <= 16 ? launch_paged_merge_few(dtype, a, s) : launch_paged_merge(dtype, a, s);
}

}  // namespace esp
