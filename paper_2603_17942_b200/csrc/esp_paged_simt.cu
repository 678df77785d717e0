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
    MergeDesc desc;
    desc.parts = 0;
    if (!deal<CK>(a, blockIdx.x, tid & 31, share, c)) {
        if (tid == 0) a.desc[blockIdx.x] = desc;
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
                if (pos < c.s.kv) {
                    const int index = pos / a.pages.page_size;
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
        if (pc.slot >= 0 && pc.c0 == c.x.c0) desc = make_desc(a, c, share, pc, blockIdx.x);
        u += pc.n;
        if (u < end) next_tile<CK>(a, c);
    }
    if (tid == 0) a.desc[blockIdx.x] = desc;
}

// The tile whose first piece CTA c has as its last one (c = blockIdx.x), if other CTAs have the rest: the partials are weighed by 2^(m - max m) in the
// order of the CTAs.  A lane takes four quads of one pair; a warp has LP pairs side by side, as the partials lie.
constexpr int MERGE_WARPS = 8, MERGE_QUADS = 4, MERGE_PARTS = 4;

template <typename T, int D>
__global__ void __launch_bounds__(MERGE_WARPS * 32) k_paged_merge(const __grid_constant__ PagedAttnArgs a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x;
    const int LP = min(32, a.pairs), LQ = 32 / LP, WQ = LQ * MERGE_QUADS;       // pairs and quads side by side, quads of a warp
    const int cols = (D / 4 + WQ - 1) / WQ;                                     // warps for the quads of a pair
    const int task = blockIdx.y * MERGE_WARPS + warp, pr = (task / cols) * LP + lane % LP, q0 = (task % cols) * WQ + lane / LP;
    pdl_wait();
    const int4 dd = __ldcg(reinterpret_cast<const int4*>(a.desc + c));
    const int token = dd.x, n_pairs = dd.y, head0 = dd.z, n = dd.w >> 1, first_slot = dd.w & 1;
    if (n == 0 || pr >= n_pairs || q0 >= D / 4) return;
    // CTA c has the tile's first piece in slot 0 if the tile is where it starts; the CTAs behind it have theirs in slot 0
    const float2* ml = a.part_ml + part_row(a, c, 0, pr);
    // (loads of several parts are under way at once: a part at a time, every one is a round trip)
    auto slot_of = [&](int k) { return 2 * k + (k == 0 ? first_slot : 0); };
    float m = -INFINITY;
    for (int k0 = 0; k0 < n; k0 += 8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __ldcg(ml + (size_t)slot_of(min(k0 + e, n - 1)) * a.pairs).x;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, x[e]);
    }
    const float m_use = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    float4 o[MERGE_QUADS];
#pragma unroll
    for (int i = 0; i < MERGE_QUADS; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    const size_t part = (size_t)(D / 4) * a.pairs;
    const float4* po = a.part_o + part_quad(a, c, 0, q0, pr);
    for (int k0 = 0; k0 < n; k0 += MERGE_PARTS) {
        float2 x[MERGE_PARTS];
        float4 v[MERGE_PARTS][MERGE_QUADS];
#pragma unroll
        for (int e = 0; e < MERGE_PARTS; ++e) {
            const int sl = slot_of(min(k0 + e, n - 1));
            x[e] = __ldcg(ml + (size_t)sl * a.pairs);
#pragma unroll
            for (int i = 0; i < MERGE_QUADS; ++i) v[e][i] = __ldcg(po + sl * part + (q0 + i * LQ < D / 4 ? i * LQ : 0) * a.pairs);
        }
#pragma unroll
        for (int e = 0; e < MERGE_PARTS; ++e) {
            if (k0 + e >= n) break;
            const float w = exp2f(x[e].x - m_use);
            l = fmaf(x[e].y, w, l);
#pragma unroll
            for (int i = 0; i < MERGE_QUADS; ++i) {
                o[i].x = fmaf(v[e][i].x, w, o[i].x); o[i].y = fmaf(v[e][i].y, w, o[i].y);
                o[i].z = fmaf(v[e][i].z, w, o[i].z); o[i].w = fmaf(v[e][i].w, w, o[i].w);
            }
        }
    }
    const int row = pr / a.group, head = head0 + pr - row * a.group;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* y = reinterpret_cast<T*>(a.out.p) + out_offset(a.out, token + row, head);
#pragma unroll
    for (int i = 0; i < MERGE_QUADS; ++i) {
        const int q = q0 + i * LQ;
        if (q < D / 4) store4<T>(y + 4 * q, make_float4(o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv), a.out_vec);
    }
    if (a.lse && q0 == 0) a.lse[(size_t)(token + row) * a.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
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
    const int lp = a.pairs < 32 ? a.pairs : 32, wq = 32 / lp * MERGE_QUADS;
    const int tasks = (a.rows * a.group + lp - 1) / lp * ((D / 4 + wq - 1) / wq);
    if (a.n_cta < 2) return 0;
    return launch_k(k_paged_merge<T, D>, dim3(a.n_cta - 1, (tasks + MERGE_WARPS - 1) / MERGE_WARPS), dim3(MERGE_WARPS * 32), 0, s, true, a) != cudaSuccess;
}

}  // namespace

int launch_paged_merge(int dtype, const PagedAttnArgs& a, cudaStream_t s) {
    if (dtype == 0) return a.D == 32 ? run_merge<float, 32>(a, s) : (a.D == 64 ? run_merge<float, 64>(a, s) : run_merge<float, 128>(a, s));
    return a.D == 32 ? run_merge<__nv_bfloat16, 32>(a, s) : (a.D == 64 ? run_merge<__nv_bfloat16, 64>(a, s) : run_merge<__nv_bfloat16, 128>(a, s));
}

int launch_paged_simt(int dtype, PagedAttnArgs a, int n_sm, cudaStream_t s) {
    const int need = a.group * a.seq.max_new;       // pairs of the longest sequence and KV head
    a.pairs = need <= 16 ? 16 : 64;
    a.rows = a.pairs / a.group;
    if (a.rows < 1) return -1;                      // more than 64 query heads share a KV head
    a.n_cta = n_sm * (a.pairs == 16 ? 4 : 2);
    a.min_units = 2;
    const int rc = dtype == 0 ? run_simt_t<float>(a, s) : run_simt_t<__nv_bfloat16>(a, s);
    if (rc) return rc;
    return a.pairs <= 16 ? launch_paged_merge_few(dtype, a, s) : launch_paged_merge(dtype, a, s);
}

}  // namespace esp
