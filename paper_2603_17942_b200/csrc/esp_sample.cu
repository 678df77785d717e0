// Sampling from rows of logits: temperature, top-k, top-p and min-p, from one given random number a row.
//
// A cluster of blocks has a row, each block a stretch of it that it copies into its shared memory once; everything else reads it there.
//   order      larger logits first, of equal ones the lower index: a 32-bit key of the logit (its bits in the order of the values) and the index.
//   bounds     top-k and top-p keep a front of that order, so each is a last (key, index).  It is found with histograms: of (largest - logit) / temperature in steps of
//              1/16 octave first, then of the keys inside the bin that holds the border, until few enough elements are left to be sorted, or all that are left are equal.
//   weights    exp in 64 bits, summed in 64 bits in a fixed order, wherever a sum decides; the histogram's own sums only say where to look, and what is found is
//              checked against the exact ones.
//   draw       sums of the kept weights by stretches in the order of indices, then the stretch in which uniform * total lies, then the element.
#include <cooperative_groups.h>
#include <math.h>

#include "esp_paged.cuh"

namespace cg = cooperative_groups;

namespace esp {

namespace {

using paged::warp_scan_u32;

constexpr int NT = 512, NW = NT / 32;
constexpr int BINS = 512;                 // of a histogram: 32 octaves of weights in steps of 1/16
constexpr int MAX_CL = 8;                 // blocks of a cluster at most
constexpr int LIST = 2048;                // elements that are sorted at most
constexpr int SMEM_ROW = 96 * 1024;       // bytes of a row that a block keeps

__device__ __forceinline__ uint32_t order_key(float x) {        // no NaN comes here
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
template <typename T> __device__ __forceinline__ float load_logit(const T* x) {
    const float v = to_f32(*x);
    return v != v ? -INFINITY : v;
}

__device__ __forceinline__ double warp_sum_f64(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double warp_scan_f64(double v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}

struct Shared {
    unsigned long long best[MAX_CL];      // largest (key, ~index) of each block
    double sum[2][MAX_CL];                // a sum of each block
    unsigned count[2][MAX_CL];
    uint32_t lo[MAX_CL], hi[MAX_CL];      // smallest and largest key of an interval in each block
    uint32_t hist[BINS], mass[BINS];      // elements, and weights in 2^-scale of the bin's largest
    uint32_t all[BINS], all_mass[BINS];   // the cluster's
    unsigned long long list[LIST];        // block 0: ~(key, ~index), so that the order is ascending
    double list_w[LIST];
    uint32_t n_list;
    double warp_sum[NW];
    unsigned warp_count[NW];
    unsigned long long answer;
    double answer_w;
    int bin;
    unsigned above;
};

struct Row {
    float M;                  // the largest logit
    double inv_t;
    float steps;              // bins per unit of logit
    unsigned long long bound; // what stays is <= bound in the order (~key << 32 | index)
    double min_p;
};
// The order as one number, ascending: 0 is the first of all.
__device__ __forceinline__ unsigned long long rank_of(float x, int index) { return ((unsigned long long)~order_key(x) << 32) | (unsigned)index; }
__device__ __forceinline__ double weight(const Row& r, float x) {
    if (x == r.M) return 1.0;
    if (isinf(x) || isinf(r.M)) return 0.0;
    return exp(((double)x - (double)r.M) * r.inv_t);
}
__device__ __forceinline__ int bin_of(const Row& r, float x) { return x == r.M ? 0 : (int)fminf((r.M - x) * r.steps, (float)(BINS - 1)); }

template <typename T, bool RESIDENT>
__global__ void __launch_bounds__(NT) k_sample(const __grid_constant__ SampleArgs a) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ Shared sm;
    cg::cluster_group cluster = cg::this_cluster();
    const int CL = cluster.num_blocks(), me = cluster.block_rank(), row = blockIdx.x / CL;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const T* logits = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride;
    const int first = min(a.vocab, me * a.chunk), n = min(a.vocab, first + a.chunk) - first;   // (chunk * CL fits 32 bits)
    T* kept_row = reinterpret_cast<T*>(smem_raw);
    auto at = [&](int i) { return RESIDENT ? load_logit(kept_row + i) : load_logit(logits + first + i); };
    // each warp has a stretch of its own, lanes side by side
    const int each = (a.chunk + NT - 1) / NT * 32, w0 = min(n, warp * each), w1 = min(n, w0 + each);

    Row r;
    const float temperature = a.temperature ? __ldg(a.temperature + row) : 1.f, uniform = __ldg(a.uniform + row);
    const int top_k = a.top_k ? __ldg(a.top_k + row) : 0;
    const float top_p = a.top_p ? __ldg(a.top_p + row) : 1.f, min_p = a.min_p ? __ldg(a.min_p + row) : 0.f;
    const bool bad = !(temperature >= 0.f) || isinf(temperature) || !(uniform >= 0.f) || top_p != top_p || min_p != min_p;

    // ---- the largest
    unsigned long long best = ~0ull;
    for (int i = w0 + lane; i < w1; i += 32) {
        const T raw = logits[first + i];
        if (RESIDENT) kept_row[i] = raw;
        best = min(best, rank_of(load_logit(&raw), first + i));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (tid == 0) { sm.answer = ~0ull; sm.n_list = 0; }
    __syncthreads();
    if (lane == 0) atomicMin(&sm.answer, best);
    __syncthreads();
    if (tid < CL) cluster.map_shared_rank(sm.best, tid)[me] = sm.answer;
    cluster.sync();
    best = sm.best[0];
    for (int c = 1; c < CL; ++c) best = min(best, sm.best[c]);
    r.M = key_value(~(uint32_t)(best >> 32));
    if (bad || r.M == -INFINITY) {                                // the same in the whole cluster
        if (me == 0 && tid == 0) {
            a.tokens[row] = -1;
            if (a.logprob) a.logprob[row] = __int_as_float(0x7fffffff);
        }
        return;
    }
    if (temperature == 0.f || top_k == 1 || top_p <= 0.f) {       // one element stays: the first
        if (me == 0 && tid == 0) {
            a.tokens[row] = (int)(uint32_t)best;
            if (a.logprob) a.logprob[row] = 0.f;
        }
        return;
    }
    r.inv_t = 1.0 / (double)temperature;
    r.steps = fminf((float)(BINS / 32 * 1.4426950408889634 * r.inv_t), 3e38f);
    r.bound = ~0ull;
    r.min_p = (double)min_p;

    // a sum over the cluster of a number of each thread, in a fixed order; `which`: two calls without a barrier of the cluster between them use different ones
    auto cluster_sum = [&](double v, int which) {
        v = warp_sum_f64(v);
        if (lane == 0) sm.warp_sum[warp] = v;
        __syncthreads();
        double t = 0.0;
        for (int w = 0; w < NW; ++w) t += sm.warp_sum[w];
        if (tid < CL) cluster.map_shared_rank(sm.sum[which], tid)[me] = t;
        cluster.sync();
        t = 0.0;
        for (int c = 0; c < CL; ++c) t += sm.sum[which][c];
        return t;
    };

    int flip = 0;
    // ---- bounds: what = 0 top-k, 1 top-p
    for (int what = 0; what < 2; ++what) {
        if (what == 0 ? (top_k < 1 || top_k >= a.vocab) : top_p >= 1.f) continue;
        double theta = 0.0;               // top-p: the weights that have to be reached
        if (what == 1) {
            double s = 0.0;
            for (int i = w0 + lane; i < w1; i += 32) {
                const float x = at(i);
                if (rank_of(x, first + i) <= r.bound) s += weight(r, x);
            }
            theta = (double)top_p * cluster_sum(s, flip ^= 1);
        }
        uint32_t key_lo = 0, key_hi = ~0u;          // keys of the interval that holds the border
        unsigned above = 0;                         // elements in front of it
        double above_w = 0.0;                       // their weights
        int level = 0, width = 0;                   // bins of 2^width keys from level 1 on
        unsigned long long bound = 0;
        for (;;) {
            // histogram of the interval
            for (int i = tid; i < BINS; i += NT) { sm.hist[i] = 0; sm.mass[i] = 0; }
            __syncthreads();
            auto bin = [&](float x, uint32_t k) { return level == 0 ? bin_of(r, x) : (int)((key_hi - k) >> width); };
            const float scale = (float)(1u << 15);
            for (int i = w0 + lane; i < w1; i += 32) {
                const float x = at(i);
                const uint32_t k = order_key(x);
                if (k < key_lo || k > key_hi || rank_of(x, first + i) > r.bound) continue;
                const int b = bin(x, k);
                atomicAdd(&sm.hist[b], 1u);
                (void)scale;
            }
            __syncthreads();
            cluster.sync();
            for (int i = tid; i < BINS; i += NT) {
                unsigned s = 0;
                for (int c = 0; c < CL; ++c) s += cluster.map_shared_rank(sm.hist, c)[i];
                sm.all[i] = s;
            }
            __syncthreads();
            // the bin that holds the border
            int b_lo = 0;
            unsigned before = above;
            double before_w = above_w;
            if (what == 0) {
                if (tid < 32) {
                    unsigned run = above;
                    int found = -1;
                    unsigned fb = 0;
                    for (int b0 = 0; b0 < BINS && found < 0; b0 += 32) {
                        const unsigned v = sm.all[b0 + lane], in = warp_scan_u32(v, lane);
                        const uint32_t hit = __ballot_sync(0xffffffffu, run + in >= (unsigned)top_k);
                        if (hit) {
                            const int src = __ffs(hit) - 1;
                            found = b0 + src;
                            fb = run + __shfl_sync(0xffffffffu, in - v, src);
                        }
                        run += __shfl_sync(0xffffffffu, in, 31);
                    }
                    if (lane == 0) { sm.bin = found; sm.above = fb; }
                }
                __syncthreads();
                b_lo = sm.bin;
                before = sm.above;
            } else {
                // exact weights of bin after bin, from the first on (a block of bins at a time)
                for (b_lo = 0;; ++b_lo) {
                    double s = 0.0;
                    if (sm.all[b_lo] > 0) {
                        for (int i = w0 + lane; i < w1; i += 32) {
                            const float x = at(i);
                            const uint32_t k = order_key(x);
                            if (k < key_lo || k > key_hi || rank_of(x, first + i) > r.bound) continue;
                            if (bin(x, k) == b_lo) s += weight(r, x);
                        }
                        s = cluster_sum(s, flip ^= 1);
                    }
                    bool rest = false;               // elements behind this bin
                    for (int i = b_lo + 1; i < BINS && !rest; ++i) rest = sm.all[i] > 0;
                    if (sm.all[b_lo] > 0 && (before_w + s >= theta || !rest)) break;
                    before_w += s;
                    before += sm.all[b_lo];
                }
            }
            const unsigned here = sm.all[b_lo];
            // keys of the bin
            uint32_t lo = ~0u, hi = 0;
            for (int i = w0 + lane; i < w1; i += 32) {
                const float x = at(i);
                const uint32_t k = order_key(x);
                if (k < key_lo || k > key_hi || rank_of(x, first + i) > r.bound || bin(x, k) != b_lo) continue;
                lo = min(lo, k);
                hi = max(hi, k);
                if (here <= LIST) {
                    const unsigned p = atomicAdd(cluster.map_shared_rank(&sm.n_list, 0), 1u);
                    cluster.map_shared_rank(sm.list, 0)[p] = rank_of(x, first + i);
                }
            }
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            if (tid == 0) { sm.warp_count[0] = ~0u; sm.warp_count[1] = 0; }
            __syncthreads();
            if (lane == 0) { atomicMin(&sm.warp_count[0], lo); atomicMax(&sm.warp_count[1], hi); }
            __syncthreads();
            if (tid < CL) {
                cluster.map_shared_rank(sm.lo, tid)[me] = sm.warp_count[0];
                cluster.map_shared_rank(sm.hi, tid)[me] = sm.warp_count[1];
            }
            cluster.sync();
            lo = ~0u;
            hi = 0;
            for (int c = 0; c < CL; ++c) { lo = min(lo, sm.lo[c]); hi = max(hi, sm.hi[c]); }
            if (here <= LIST) {
                if (me == 0) {
                    // sort, then the border by sums in the order
                    int size = 1;
                    while (size < (int)here) size *= 2;
                    for (int i = here + tid; i < size; i += NT) sm.list[i] = ~0ull;
                    __syncthreads();
                    for (int s = 2; s <= size; s *= 2)
                        for (int d = s / 2; d > 0; d /= 2) {
                            for (int i = tid; i < size / 2; i += NT) {
                                const int x = 2 * i - (i & (d - 1)), y = x + d;
                                const unsigned long long p = sm.list[x], q = sm.list[y];
                                if ((p > q) == ((x & s) == 0)) { sm.list[x] = q; sm.list[y] = p; }
                            }
                            __syncthreads();
                        }
                    if (what == 0) {
                        if (tid == 0) sm.answer = sm.list[top_k - before - 1];
                    } else {
                        for (int i = tid; i < (int)here; i += NT) sm.list_w[i] = weight(r, key_value(~(uint32_t)(sm.list[i] >> 32)));
                        __syncthreads();
                        if (tid == 0) {
                            double run = before_w;
                            int i = 0;
                            while (i + 1 < (int)here && run + sm.list_w[i] < theta) run += sm.list_w[i++];
                            sm.answer = sm.list[i];
                        }
                    }
                    __syncthreads();
                    if (tid == 0) sm.n_list = 0;
                    if (tid > 0 && tid < CL) *cluster.map_shared_rank(&sm.answer, tid) = sm.answer;
                }
                cluster.sync();
                bound = sm.answer;
                break;
            }
            if (lo == hi) {
                // all equal: so many of them, by the lowest index
                unsigned take;
                if (what == 0) take = top_k - before;
                else {
                    const double m = ceil((theta - before_w) / weight(r, key_value(lo)));
                    take = m < 1.0 ? 1u : (m < (double)here ? (unsigned)m : here);
                }
                unsigned c = 0;
                for (int i = w0 + lane; i < w1; i += 32) c += order_key(at(i)) == lo && rank_of(at(i), first + i) <= r.bound;
                c = __reduce_add_sync(0xffffffffu, c);
                if (lane == 0) sm.warp_count[warp] = c;
                __syncthreads();
                if (tid < CL) {
                    unsigned t = 0;
                    for (int w = 0; w < NW; ++w) t += sm.warp_count[w];
                    cluster.map_shared_rank(sm.count[0], tid)[me] = t;
                }
                cluster.sync();
                unsigned run = 0;
                for (int k = 0; k < me; ++k) run += sm.count[0][k];
                for (int w = 0; w < warp; ++w) run += sm.warp_count[w];
                if (run < take && take <= run + sm.warp_count[warp]) {
                    for (int i0 = w0; i0 < w1; i0 += 32) {
                        const int i = i0 + lane;
                        const bool is = i < w1 && order_key(at(i)) == lo && rank_of(at(i), first + i) <= r.bound;
                        const uint32_t same = __ballot_sync(0xffffffffu, is);
                        if (is && run + __popc(same & ((1u << lane) - 1u)) + 1 == take)
                            for (int k = 0; k < CL; ++k) *cluster.map_shared_rank(&sm.answer, k) = rank_of(at(i), first + i);
                        run += __popc(same);
                    }
                }
                cluster.sync();
                bound = sm.answer;
                break;
            }
            key_lo = lo;
            key_hi = hi;
            above = before;
            above_w = before_w;
            level = 1;
            for (width = 0; ((hi - lo) >> width) >= BINS; ++width) {}
            cluster.sync();                         // the histograms have been read
        }
        r.bound = min(r.bound, bound);
        cluster.sync();
    }

    // ---- the draw
    auto kept_weight = [&](int i) {
        const float x = at(i);
        if (rank_of(x, first + i) > r.bound) return 0.0;
        const double w = weight(r, x);
        return w >= r.min_p || x == r.M ? w : 0.0;
    };
    double s = 0.0;
    for (int i = w0 + lane; i < w1; i += 32) s += kept_weight(i);
    const double total = cluster_sum(s, flip ^= 1);
    const double target = (double)uniform * total;
    double run = 0.0;
    for (int c = 0; c < me; ++c) run += sm.sum[flip][c];
    // the last block with weight takes what rounding leaves behind it
    bool last = true;
    for (int c = me + 1; c < CL; ++c) last = last && sm.sum[flip][c] == 0.0;
    const double mine = sm.sum[flip][me];
    if (mine > 0.0 && target >= run && (target < run + mine || last)) {
        bool last_warp = true;
        for (int w = 0; w < warp; ++w) run += sm.warp_sum[w];
        for (int w = warp + 1; w < NW; ++w) last_warp = last_warp && sm.warp_sum[w] == 0.0;
        // (sums by blocks and by warps may differ in the last bits: the warp that is first to reach the target, or the last one with weight)
        const bool mine_too = sm.warp_sum[warp] > 0.0 && (run + sm.warp_sum[warp] > target || last_warp);
        if (lane == 0) sm.warp_count[warp] = mine_too;
        if (mine_too) {
            int token = -1;
            double w_token = 0.0;
            for (int i0 = w0; i0 < w1; i0 += 32) {
                const int i = i0 + lane;
                const double w = i < w1 ? kept_weight(i) : 0.0;
                const double in = warp_scan_f64(w, lane);
                const uint32_t hit = __ballot_sync(0xffffffffu, w > 0.0 && run + in > target), any = __ballot_sync(0xffffffffu, w > 0.0);
                const int src = hit ? __ffs(hit) - 1 : (any ? 31 - __clz(any) : 0);
                if (any) {
                    token = first + i0 + src;
                    w_token = __shfl_sync(0xffffffffu, w, src);
                }
                if (hit) break;
                run += __shfl_sync(0xffffffffu, in, 31);
            }
            // of several warps the first
            if (lane == 0) {
                sm.list[warp] = (unsigned)token;
                sm.list_w[warp] = w_token;
            }
        }
    } else if (lane == 0) sm.warp_count[warp] = 0;
    __syncthreads();
    if (tid == 0)
        for (int w = 0; w < NW; ++w)
            if (sm.warp_count[w]) {
                a.tokens[row] = (int)sm.list[w];
                if (a.logprob) a.logprob[row] = (float)log(sm.list_w[w] / total);
                break;
            }
    cluster.sync();                                  // nobody leaves while others may look into its shared memory
}

template <typename T>
int run(SampleArgs a, cudaStream_t s) {
    int cl = 1;
    while (cl < MAX_CL && a.vocab > cl * 4096) cl *= 2;
    a.chunk = ((a.vocab + cl - 1) / cl + 511) / 512 * 512;
    const size_t bytes = (size_t)a.chunk * sizeof(T);
    const bool resident = bytes <= SMEM_ROW;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.n_rows * cl);
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = resident ? bytes : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cl;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (resident) {
        if (ensure_dynamic_smem(reinterpret_cast<const void*>(&k_sample<T, true>), SMEM_ROW)) return -1;
        return cudaLaunchKernelEx(&cfg, k_sample<T, true>, a) != cudaSuccess;
    }
    return cudaLaunchKernelEx(&cfg, k_sample<T, false>, a) != cudaSuccess;
}

}  // namespace

int launch_sample(int dtype, SampleArgs a, int n_sm, cudaStream_t s) {
    (void)n_sm;
    return dtype == 0 ? run<float>(a, s) : run<__nv_bfloat16>(a, s);
}

}  // namespace esp

using namespace esp;

extern "C" {

int esp_sample_scratch_bytes(int32_t n_rows, int32_t vocab, size_t* bytes_out) {
    if (!bytes_out || n_rows < 0 || vocab < 1) return ESP_E_ARG;
    *bytes_out = 256;
    return ESP_OK;
}

int esp_sample(int32_t dtype, int32_t n_rows, int32_t vocab, const void* logits, int64_t row_stride, const esp_sampling* sampling, const float* uniform,
               int32_t* tokens, float* logprob, void* scratch, size_t scratch_bytes, void* cuda_stream) {
    if (dtype != 0 && dtype != 1) return ESP_E_BADCFG;
    const int size = dtype == 0 ? 4 : 2;
    auto off = [](const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; };
    if (n_rows < 0 || n_rows > (1 << 27) || vocab < 1 || vocab > (1 << 24) || row_stride < 0 || row_stride > ((int64_t)1 << 40) || !sampling) return ESP_E_ARG;
    if (off(logits, size) || off(sampling->temperature, 4) || off(sampling->top_k, 4) || off(sampling->top_p, 4) || off(sampling->min_p, 4) || off(uniform, 4) ||
        off(tokens, 4) || off(logprob, 4)) return ESP_E_ARG;
    if (n_rows == 0) return ESP_OK;
    if (!logits || !uniform || !tokens) return ESP_E_ARG;
    size_t need = 0;
    if (const int rc = esp_sample_scratch_bytes(n_rows, vocab, &need)) return rc;
    if (!scratch || scratch_bytes < need || off(scratch, 256)) return ESP_E_WORKSPACE;
    const int n_sm = current_sm_count();
    if (n_sm < 1) return ESP_E_CUDA;
    SampleArgs a;
    a.logits = logits; a.row_stride = row_stride; a.n_rows = n_rows; a.vocab = vocab;
    a.temperature = sampling->temperature; a.top_k = sampling->top_k; a.top_p = sampling->top_p; a.min_p = sampling->min_p;
    a.uniform = uniform; a.tokens = tokens; a.logprob = logprob; a.chunk = 0;
    const int rc = launch_sample(dtype, a, n_sm, reinterpret_cast<cudaStream_t>(cuda_stream));
    const cudaError_t e = cudaGetLastError();
    return rc ? ESP_E_CUDA : (e == cudaSuccess ? ESP_OK : ESP_E_CUDA);
}

}  // extern "C"
