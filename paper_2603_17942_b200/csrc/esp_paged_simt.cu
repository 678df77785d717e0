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
    Deal deal;
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
    if (!deal<CK, false>(a, blockIdx.x, 1, &sm.deal)) return;
    Cursor c = sm.deal.at;
    const long long total = sm.deal.total, begin = sm.deal.unit, end = cta_begin(total, sm.deal.ctas, blockIdx.x + 1);
    const bool dims = D >= 64 || tx < 8;

    for (long long u = begin; u < end;) {
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
                    for (int j = 0; j < DV; ++j) {
                        T* z = y + tx * 4 + 64 * j;
                        z[0] = from_f32<T>(o[i][j].x * inv); z[1] = from_f32<T>(o[i][j].y * inv);
                        z[2] = from_f32<T>(o[i][j].z * inv); z[3] = from_f32<T>(o[i][j].w * inv);
                    }
                if (a.lse && tx == 0) a.lse[(size_t)token * a.Hq + head] = l_run[i] == 0.f ? -INFINITY : (m_run[i] + log2f(l_run[i])) * 0.6931471805599453f;
            } else {
                const size_t at = ((size_t)blockIdx.x * 2 + pc.slot) * a.pairs + pr;
                if (dims)
#pragma unroll
                    for (int j = 0; j < DV; ++j) *reinterpret_cast<float4*>(a.part_o + at * D + tx * 4 + 64 * j) = o[i][j];
                if (tx == 0) a.part_ml[at] = make_float2(m_run[i], l_run[i]);
            }
        }
        u += pc.n;
        if (u < end) next_tile<CK>(a, c);
    }
}

// Block (c, slice): the tile whose first piece CTA c has as its last one, if other CTAs have the rest; a warp per pair, which weighs
// the partials by 2^(m - max m) in the order of the CTAs.  The dealing is looked up while the kernel in front still runs.
constexpr int MERGE_WARPS = 8;

template <typename T, int D, int CKM>
__global__ void __launch_bounds__(MERGE_WARPS * 32) k_paged_merge(const __grid_constant__ PagedAttnArgs a, int min_units) {
    __shared__ Deal sd;
    const int c = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool any = deal<CKM, true>(a, c, min_units, &sd);
    const Cursor& t = sd.at;
    const bool split = any && t.tile_u >= cta_begin(sd.total, sd.ctas, c) && t.tile_u + t.x.nc > cta_begin(sd.total, sd.ctas, c + 1);
    pdl_wait();
    if (!split) return;
    const int c_last = cta_of_unit(sd.total, sd.ctas, t.tile_u + t.x.nc - 1);
    // CTA c has the tile's first piece in slot 0 if the tile is where it starts; the CTAs behind it have theirs in slot 0
    const int first_slot = cta_begin(sd.total, sd.ctas, c) >= t.tile_u ? 0 : 1;
    const int n_pairs = t.x.nr * a.group;
    for (int pr = blockIdx.y * MERGE_WARPS + warp; pr < n_pairs; pr += gridDim.y * MERGE_WARPS) {
        auto at = [&](int cta) { return ((size_t)cta * 2 + (cta == c ? first_slot : 0)) * a.pairs + pr; };
        float m = -INFINITY;
        for (int k = c + lane; k <= c_last; k += 32) m = fmaxf(m, __ldcg(a.part_ml + at(k)).x);
        m = warp_max(m);
        const float m_use = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        float o[D / 32];
#pragma unroll
        for (int i = 0; i < D / 32; ++i) o[i] = 0.f;
        for (int k0 = c; k0 <= c_last; k0 += 32) {
            float w = 0.f, lk = 0.f;
            if (k0 + lane <= c_last) {
                const float2 ml = __ldcg(a.part_ml + at(k0 + lane));
                w = exp2f(ml.x - m_use);
                lk = ml.y * w;
            }
            const int n = min(32, c_last - k0 + 1);
#pragma unroll 4
            for (int j = 0; j < n; ++j) {
                const float wj = __shfl_sync(0xffffffffu, w, j);
                l += __shfl_sync(0xffffffffu, lk, j);
                const float* src = a.part_o + at(k0 + j) * D + lane * (D / 32);
                float x[D / 32];
                if constexpr (D == 128) {
                    const float4 y = __ldcg(reinterpret_cast<const float4*>(src));
                    x[0] = y.x; x[1] = y.y; x[2] = y.z; x[3] = y.w;
                } else if constexpr (D == 64) {
                    const float2 y = __ldcg(reinterpret_cast<const float2*>(src));
                    x[0] = y.x; x[1] = y.y;
                } else {
                    x[0] = __ldcg(src);
                }
#pragma unroll
                for (int i = 0; i < D / 32; ++i) o[i] = fmaf(wj, x[i], o[i]);
            }
        }
        const int row = pr / a.group, head = t.kvh * a.group + pr - row * a.group, token = t.s.start + t.x.r0 + row;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* y = reinterpret_cast<T*>(a.out.p) + out_offset(a.out, token, head) + lane * (D / 32);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) y[i] = from_f32<T>(o[i] * inv);
        if (a.lse && lane == 0) a.lse[(size_t)token * a.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
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

template <typename T, int D, int CKM>
int run_merge(const PagedAttnArgs& a, int min_units, cudaStream_t s) {
    const int slices = (a.rows * a.group + MERGE_WARPS - 1) / MERGE_WARPS;
    if (a.n_cta < 2) return 0;
    return launch_k(k_paged_merge<T, D, CKM>, dim3(a.n_cta - 1, slices), dim3(MERGE_WARPS * 32), 0, s, true, a, min_units) != cudaSuccess;
}
template <typename T, int CKM>
int run_merge_d(const PagedAttnArgs& a, int min_units, cudaStream_t s) {
    return a.D == 32 ? run_merge<T, 32, CKM>(a, min_units, s) : (a.D == 64 ? run_merge<T, 64, CKM>(a, min_units, s) : run_merge<T, 128, CKM>(a, min_units, s));
}

}  // namespace

int launch_paged_merge(int dtype, const PagedAttnArgs& a, int chunk, int min_units, cudaStream_t s) {
    if (dtype == 0) return run_merge_d<float, CK>(a, min_units, s);
    return chunk == 64 ? run_merge_d<__nv_bfloat16, 64>(a, min_units, s) : run_merge_d<__nv_bfloat16, 128>(a, min_units, s);
}

int launch_paged_simt(int dtype, PagedAttnArgs a, int n_sm, cudaStream_t s) {
    const int need = a.group * a.seq.max_new;       // pairs of the longest sequence and KV head
    a.pairs = need <= 16 ? 16 : 64;
    a.rows = a.pairs / a.group;
    if (a.rows < 1) return -1;                      // more than 64 query heads share a KV head
    a.n_cta = n_sm * (a.pairs == 16 ? 4 : 2);
    const int rc = dtype == 0 ? run_simt_t<float>(a, s) : run_simt_t<__nv_bfloat16>(a, s);
    return rc ? rc : launch_paged_merge(dtype, a, CK, 1, s);
}

}  // namespace esp
