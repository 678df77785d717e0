// Weights of cached positions on CUDA cores (fp32, and bf16 where the tensor-core kernels do not take the head size, page size or alignment), and
// the join of chunks that several CTAs share.
//
// A block holds a chunk of 64 keys in shared memory as fp32 and walks the tiles of 32 (token, query head) pairs that see it: thread (ty, tx), 16 x 16, has
// pairs 2 ty and 2 ty + 1 and keys tx + 16 j.  The weights exp(scale q k - lse) add up in registers, one number for each of a thread's keys, and over the ty at the end.
// Shared memory bounds long calls: for four elements of a head a warp reads six float4, about 10 cycles of its pipe, for multiply-adds that take the SM 8 (fp32, 4 x 1000 tokens, 8/2 heads of
// 128: 190 us, 22 TFLOP/s, the pipe busy for 85 % of the cycles and the multiply-adds' for 41 %; with one block an SM 322).  The chain from lengths over pages to keys bounds small ones (6 to 10 us).
#include "esp_key_weights.cuh"

namespace esp {

namespace {

using namespace paged;

constexpr int CK = 64, MP = 32, THREADS = 256;
constexpr int BLOCKS = KEY_WEIGHT_KEYS / CK;      // of an SM: as many as the scratch has room for

template <int D>
struct Smem {
    float q[MP][D + 4];
    float k[CK][D + 4];
    float sum[16][CK];
    float lse[MP];
    long long base[CK];
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

template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(THREADS, BLOCKS) k_key_weights_simt(const __grid_constant__ KeyWeightArgs w) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem_raw);
    const PagedAttnArgs& a = w.a;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    pdl_launch_dependents();
    Share share;
    WCursor c;
    if (!deal_keys<CK>(w, blockIdx.x, tid & 31, share, c)) return;
    const uint32_t begin = share.begin(blockIdx.x), end = share.begin(blockIdx.x + 1);
    for (uint32_t u = begin; u < end;) {
        const WPiece pc = make_piece(c, begin, u, end);
        const Seq& s = c.x.s;
        const int L = s.kv - s.n, p0 = c.c * CK;
        // what no token of the piece sees is not looked up: a server may have given its pages back
        const int lo = a.window > 0 ? L + c.x.i0 + pc.t0 * a.rows - a.window + 1 : 0;
        __syncthreads();
        if (tid < CK) {
            const int pos = p0 + tid;
            long long base = -1;
            if (pc.n > 0 && pos < s.kv && pos >= lo) {
                const int index = page_index(a.pages, pos), page = load_page(a.seq, a.pages, c.b, index);
                if (page >= 0) base = page * a.pages.page + (pos - index * a.pages.page_size) * a.pages.tok + c.kvh * a.pages.head;
            }
            sm.base[tid] = base;
        }
        __syncthreads();
        {
            constexpr int N = CK * (D / 4) / THREADS;        // all of a thread's loads under way
            float4 x[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int i = tid + j * THREADS, r = i / (D / 4), d = (i % (D / 4)) * 4;
                x[j] = sm.base[r] >= 0 ? load4<T, VEC>(reinterpret_cast<const T*>(a.pages.k) + sm.base[r] + d) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int i = tid + j * THREADS;
                *reinterpret_cast<float4*>(&sm.k[i / (D / 4)][(i % (D / 4)) * 4]) = x[j];
            }
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        for (int t = pc.t0; t < pc.t0 + pc.n; ++t) {
            const int r0 = c.x.i0 + t * a.rows, n_pairs = min(a.rows, s.n - r0) * a.group;
            // a tile of more pairs than the block takes at a time: part after part
            for (int part = 0; part < n_pairs; part += MP) {
                __syncthreads();
                for (int i = tid; i < MP * (D / 4); i += THREADS) {
                    const int r = i / (D / 4), d = (i % (D / 4)) * 4, pr = part + r;
                    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (pr < n_pairs) {
                        const int row = pr / a.group, head = c.kvh * a.group + pr - row * a.group;
                        x = load4<T, VEC>(reinterpret_cast<const T*>(a.q.p) + out_offset(a.q, s.start + r0 + row, head) + d);
                    }
                    *reinterpret_cast<float4*>(&sm.q[r][d]) = x;
                }
                if (tid < MP) {
                    const int pr = part + tid, row = pr / a.group;
                    sm.lse[tid] = pr < n_pairs ? __ldg(w.lse + (size_t)(s.start + r0 + row) * a.Hq + c.kvh * a.group + pr - row * a.group) * 1.4426950408889634f : 0.f;
                }
                __syncthreads();
                float x[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[i][j] = 0.f;
#pragma unroll 4
                for (int d = 0; d < D; d += 4) {
                    float4 qv[2], kv[4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) qv[i] = *reinterpret_cast<const float4*>(&sm.q[ty * 2 + i][d]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4*>(&sm.k[tx + 16 * j][d]);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            x[i][j] = fmaf(qv[i].x, kv[j].x, fmaf(qv[i].y, kv[j].y, fmaf(qv[i].z, kv[j].z, fmaf(qv[i].w, kv[j].w, x[i][j]))));
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int pr = part + ty * 2 + i;
                    if (pr >= n_pairs) continue;
                    const RowMask m = row_mask(a, s, r0 + pr / a.group);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (sees(m, p0 + tx + 16 * j, L, s.kv)) sum[j] += exp2f(fmaf(x[i][j], a.scale_log2, -sm.lse[ty * 2 + i]));
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) sm.sum[ty][tx + 16 * j] = sum[j];
        __syncthreads();
        if (tid < CK && p0 + tid < s.kv) {
            float total = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) total += sm.sum[i][tid];
            if (pc.slot < 0) store_score(w, c, p0 + tid, total);
            else w.part[((size_t)blockIdx.x * 2 + pc.slot) * CK + tid] = total;
        }
        u += max(pc.n, 1);
        if (u < end) next_chunk<CK>(w, c);
    }
}

// The chunk that CTA c has the first piece of as its last one: the pieces' sums in the order of the CTAs.  (Each block deals as the CTA did.)
template <int KEYS>
__global__ void __launch_bounds__(KEYS) k_key_weights_join(const __grid_constant__ KeyWeightArgs w) {
    Share share;
    WCursor c, n;
    const int cta = blockIdx.x;
    uint32_t begin = 0, end = 0;
    bool joins = deal_keys<KEYS>(w, cta, threadIdx.x & 31, share, c) && cta + 1 < share.ctas;
    if (joins) {
        begin = share.begin(cta);
        end = share.begin(cta + 1);
        // the chunk in which the next CTA starts, if it is one that this CTA starts (otherwise nobody shares, or another CTA has the first piece)
        deal_keys<KEYS>(w, cta + 1, threadIdx.x & 31, share, n);
        joins = n.chunk_u >= begin && n.chunk_u < end;
    }
    pdl_wait();                           // by every block: who comes behind this grid has to find the sums written
    if (!joins) return;
    const int last = share.cta_of(n.chunk_u + n.k.units() - 1), pos = n.c * KEYS + threadIdx.x;
    if (pos >= n.x.s.kv) return;
    float sum = 0.f;
    for (int k = cta; k <= last; ++k) {
        const int slot = k == cta && begin < n.chunk_u ? 1 : 0;
        sum += __ldcg(w.part + ((size_t)k * 2 + slot) * KEYS + threadIdx.x);
    }
    store_score(w, n, pos, sum);
}

template <typename T, int D>
int run(const KeyWeightArgs& w, cudaStream_t s) {
    auto go = [&](auto kernel) {
        if (ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)sizeof(Smem<D>))) return -1;
        kernel<<<w.a.n_cta, THREADS, sizeof(Smem<D>), s>>>(w);
        return 0;
    };
    return w.a.vec ? go(k_key_weights_simt<T, D, true>) : go(k_key_weights_simt<T, D, false>);
}

}  // namespace

int launch_key_weights_simt(int dtype, KeyWeightArgs w, int n_sm, cudaStream_t s) {
    PagedAttnArgs& a = w.a;
    a.rows = a.group <= MP ? MP / a.group : 1;
    a.rows_shift = shift_of(a.rows);
    a.n_cta = n_sm * BLOCKS;
    a.min_units = 1;
    int rc;
    if (dtype == 0) rc = a.D == 32 ? run<float, 32>(w, s) : (a.D == 64 ? run<float, 64>(w, s) : run<float, 128>(w, s));
    else rc = a.D == 32 ? run<__nv_bfloat16, 32>(w, s) : (a.D == 64 ? run<__nv_bfloat16, 64>(w, s) : run<__nv_bfloat16, 128>(w, s));
    const int observed = w.last > 0 && w.last < a.seq.max_new ? w.last : a.seq.max_new;
    // (no chunk has two owners where all observed tokens are one tile)
    return rc || observed <= a.rows ? rc : launch_key_weights_join(w, CK, s);
}

int launch_key_weights_join(const KeyWeightArgs& w, int keys, cudaStream_t s) {
    if (w.a.n_cta < 2) return 0;
    const dim3 grid(w.a.n_cta - 1), block(keys);
    return (keys == CK ? launch_k(k_key_weights_join<CK>, grid, block, 0, s, true, w) : launch_k(k_key_weights_join<KEY_WEIGHT_KEYS>, grid, block, 0, s, true, w)) != cudaSuccess;
}

}  // namespace esp
