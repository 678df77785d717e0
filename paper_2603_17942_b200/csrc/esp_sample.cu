// Sampling from rows of logits: temperature, top-k, top-p and min-p, from one given random number a row.
//
// A cluster of blocks has a row, each block a stretch of it that it copies into its shared memory once; everything else reads it there.
//   order      larger logits first, of equal ones the lower index: a 32-bit key of the logit (its bits in the order of the values) and the index.  top-k, top-p and min-p each
//              keep a front of that order.
//   weights    exp in 64 bits, summed in 64 bits in a fixed order, wherever a sum decides.
//   list       A histogram of (largest - logit) / temperature in steps of 1/24 octave (elements, or their weights to 2e-4) says behind which bin the front ends at the latest.  What
//              lies in front of that, a few dozen to a few hundred elements, goes to the first block, the others are done.  It sorts them, takes exact sums along the order,
//              cuts, and finds the token by searching the index at which the kept weights exceed uniform times their sum.
//   otherwise  (fronts of thousands of elements, and rows without a limit): the last element of each front by histograms that close in on it, then sums of
//              the kept weights by stretches in the order of indices, the stretch in which uniform * total lies, the element.
#include <cooperative_groups.h>
#include <math.h>

#include "esp_paged.cuh"

namespace cg = cooperative_groups;

namespace esp {

namespace {

using paged::warp_scan_u32;

constexpr int NT = 512, NW = NT / 32;
constexpr int BINS = NT;                  // of a histogram, a thread for each
constexpr float STEPS = 24.f;             // bins of an octave of weights: 21 octaves
constexpr int MAX_CL = 8;                 // blocks of a cluster at most
constexpr int LIST = 2048;                // elements that are sorted at most
constexpr int SMEM_ROW = 160 * 1024;      // bytes of a row that a block keeps at most
constexpr int TAB = 256;                  // 2^(j / TAB)
constexpr float UNIT = 8192.f;            // a histogram of weights counts in 1 / UNIT of a bin's largest: 2^19 elements of a block fit 32 bits
constexpr int MAX_VOCAB = 1 << 21;

__device__ __forceinline__ uint32_t order_key(float x) {        // no NaN comes here
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ float number(float v) { return v != v ? -INFINITY : v; }

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
    double tab[TAB];
    unsigned long long best[MAX_CL];      // the first of each block
    double sum[2][MAX_CL];                // a sum of each block
    unsigned count[MAX_CL];
    uint32_t lo[MAX_CL], hi[MAX_CL];      // smallest and largest key of an interval in each block
    uint32_t hist[BINS];
    uint32_t all[BINS];                   // the cluster's
    unsigned long long list[LIST];        // the first block's
    double list_w[LIST];
    uint32_t n_list;
    double warp_sum[NW], warp_sum2[NW];
    float warp_f[NW];
    unsigned warp_count[NW];
    unsigned long long answer;
    int bin;
    unsigned above;
};

struct Row {
    float M;                  // the largest logit
    double Md, A;             // the same; TAB * log2 e / temperature
    float steps;              // bins per unit of logit
    unsigned long long bound; // what stays is <= bound in the order
    double min_p;
};
// The order as one number, ascending: 0 is the first of all.
__device__ __forceinline__ unsigned long long rank_of(float x, int index) { return ((unsigned long long)~order_key(x) << 32) | (unsigned)index; }
__device__ __forceinline__ float rank_value(unsigned long long r) { return key_value(~(uint32_t)(r >> 32)); }

// A float as a double by its bits (the conversion instruction runs at a quarter of the rate of the sums).  Zero comes out as 2^-127, infinity as 2^128.
__device__ __forceinline__ double widen(float x) {
    const uint32_t b = __float_as_uint(x);
    return __hiloint2double((int)((b & 0x80000000u) | (((b & 0x7fffffffu) >> 3) + (896u << 20))), (int)(b << 29));
}
// exp((x - M) / temperature): 2^n * 2^(j / 256) from a table * a polynomial of degree 3 on what is left, |r| <= 1/512 octave: (ln 2 / 512)^4 / 24 = 1.4e-13 of the
// weight.  Weights below 2^-60 of the largest count as nothing.
__device__ __forceinline__ double weight(const Row& r, const double* tab, float x) {
    constexpr double C1 = 0.6931471805599453 / TAB, C2 = C1 * C1 / 2, C3 = C1 * C1 * C1 / 6, MAGIC = 6755399441055744.0;
    const double t = (widen(x) - r.Md) * r.A;
    const double y = t + MAGIC;
    const int n = __double2loint(y);
    const double d = t - (y - MAGIC);
    const double p = fma(d, fma(d, fma(d, C3, C2), C1), 1.0) * tab[n & (TAB - 1)];
    const double w = __hiloint2double(__double2hiint(p) + ((n >> 8) << 20), __double2loint(p));
    return t > -60.0 * TAB && x != -INFINITY ? w : 0.0;
}
// Bins from the largest logit down; BINS - 1: somewhere behind.
__device__ __forceinline__ float depth_of(const Row& r, float x) { return x == r.M ? 0.f : fminf((r.M - x) * r.steps, (float)(BINS - 1)); }

template <typename T> struct Raw;
template <> struct Raw<float> {
    static constexpr int VEC = 4;
    __device__ static void unpack(const uint4& u, float (&x)[4]) {
        x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
    }
    __device__ static uint4 pack(const float (&x)[4]) { return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])); }
};
template <> struct Raw<__nv_bfloat16> {
    static constexpr int VEC = 8;
    __device__ static void unpack(const uint4& u, float (&x)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    __device__ static uint4 pack(const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <typename T, bool RESIDENT>
__global__ void __launch_bounds__(NT) k_sample(const __grid_constant__ SampleArgs a) {
    constexpr int VEC = Raw<T>::VEC, STRIDE = 32 * VEC;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ Shared sm;
    cg::cluster_group cluster = cg::this_cluster();
    const int CL = cluster.num_blocks(), me = cluster.block_rank(), row = blockIdx.x / CL;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const T* logits = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride;
    const int first = min(a.vocab, me * a.chunk), n = min(a.vocab, first + a.chunk) - first;   // (chunk * CL fits 32 bits)
    const bool aligned = reinterpret_cast<uintptr_t>(logits + first) % 16 == 0;
    uint4* kept_row = reinterpret_cast<uint4*>(smem_raw);
    // each warp has a stretch of its own, lanes side by side with VEC elements each
    const int each = (a.chunk / STRIDE + NW - 1) / NW * STRIDE, w0 = min(n, warp * each), w1 = min(n, w0 + each);
    // elements i .. i + VEC - 1 of the block's stretch; -infinity behind its end
    auto fetch = [&](int i, float (&x)[VEC]) {
        if (aligned && i + VEC <= n) Raw<T>::unpack(__ldg(reinterpret_cast<const uint4*>(logits + first + i)), x);
        else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = i + e < n ? to_f32(logits[first + i + e]) : -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = number(x[e]);
    };
    auto load = [&](int i, float (&x)[VEC]) {
        if (RESIDENT) Raw<T>::unpack(kept_row[i / VEC], x);
        else fetch(i, x);
    };

    Row r;
    const float temperature = a.temperature ? __ldg(a.temperature + row) : 1.f, uniform = __ldg(a.uniform + row);
    const int top_k = a.top_k ? __ldg(a.top_k + row) : 0;
    const float top_p = a.top_p ? __ldg(a.top_p + row) : 1.f, min_p = a.min_p ? __ldg(a.min_p + row) : 0.f;
    const bool bad = !(temperature >= 0.f) || isinf(temperature) || !(uniform >= 0.f) || top_p != top_p || min_p != min_p;
    const bool use_k = top_k >= 1 && top_k < a.vocab, use_p = top_p < 1.f, use_m = min_p > 0.f;

    // ---- the largest
    unsigned long long best = ~0ull;
#pragma unroll 4
    for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
        float x[VEC];
        fetch(i, x);
        if (RESIDENT) kept_row[i / VEC] = Raw<T>::pack(x);
        float m = x[0];
#pragma unroll
        for (int e = 1; e < VEC; ++e) m = fmaxf(m, x[e]);
        if (best == ~0ull || m > rank_value(best)) {
            int at = VEC - 1;
#pragma unroll
            for (int e = VEC - 2; e >= 0; --e) at = x[e] == m ? e : at;
            best = rank_of(m, first + i + at);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = min(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (tid == 0) { sm.answer = ~0ull; sm.n_list = 0; }
    if (tid < TAB) sm.tab[tid] = exp2((double)tid / TAB);
    sm.hist[tid] = 0;
    __syncthreads();
    if (lane == 0) atomicMin(&sm.answer, best);
    __syncthreads();
    if (tid < CL) cluster.map_shared_rank(sm.best, tid)[me] = sm.answer;
    cluster.sync();
    best = sm.best[0];
    for (int c = 1; c < CL; ++c) best = min(best, sm.best[c]);
    r.M = rank_value(best);
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
    const double inv_t = isinf(r.M) ? 1e300 : 1.0 / (double)temperature;      // (next to an infinite logit no other has weight)
    r.Md = widen(r.M);
    r.A = inv_t * (TAB * 1.4426950408889634);
    r.steps = (float)fmin(inv_t * ((double)STEPS * 1.4426950408889634), 3e38);
    r.bound = ~0ull;
    r.min_p = fmin((double)min_p, 1.0);

    int flip = 0;
    // a number of each thread, summed over the cluster in a fixed order; each block's share stays in sm.sum[flip], each warp's in sm.warp_sum.  Starts with publish(), and
    // after a barrier of the cluster total() has it
    auto publish = [&](double v) {
        flip ^= 1;                        // (who is still reading the last one reads the other half)
        v = warp_sum_f64(v);
        if (lane == 0) sm.warp_sum[warp] = v;
        __syncthreads();
        if (tid < CL) {
            double t = 0.0;
            for (int w = 0; w < NW; ++w) t += sm.warp_sum[w];
            cluster.map_shared_rank(sm.sum[flip], tid)[me] = t;
        }
    };
    auto total = [&]() {
        double t = 0.0;
        for (int c = 0; c < CL; ++c) t += sm.sum[flip][c];
        return t;
    };

    double S = 0.0;                       // weights of the whole row, where they count
    bool have_s = false;
    // ---- the list
    if (use_k || use_p || use_m) {
        int last_bin = BINS - 1;          // bins in front of it and it go to the list; BINS - 1: too many
        if (use_k || use_p) {
            const bool weigh = !use_k;
            double s = 0.0;
#pragma unroll 2
            for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                float x[VEC];
                load(i, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float d = depth_of(r, x[e]);
                    const int b = (int)d;
                    if (weigh) s += weight(r, sm.tab, x[e]);
                    // (2^(-1/24) = 0.97153; linear in between, off by 1.1e-4 at most)
                    if (b < BINS - 1) atomicAdd(&sm.hist[b], weigh ? (unsigned)UNIT - (unsigned)((d - (float)b) * (UNIT * (1.f - 0.97153194f))) : 1u);
                }
            }
            if (weigh) publish(s);
            cluster.sync();
            unsigned long long mine = 0;
            for (int c = 0; c < CL; ++c) mine += cluster.map_shared_rank(sm.hist, c)[tid];
            if (weigh) {
                S = total();
                have_s = true;
            }
            // sums along the bins: elements, or weights (a bin's in front of another's grow smaller by 2^(1/24))
            const float v = weigh ? (float)mine * (1.f / UNIT) * exp2f((float)tid * (-1.f / STEPS)) : (float)mine;
            float in = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float y = __shfl_up_sync(0xffffffffu, in, o);
                if (lane >= o) in += y;
            }
            const unsigned cnt = warp_scan_u32(weigh ? (unsigned)ceilf((float)mine * (1.03f / UNIT)) : (unsigned)mine, lane);
            if (lane == 31) { sm.warp_f[warp] = in; sm.warp_count[warp] = cnt; }
            if (tid == 0) sm.bin = BINS - 1;
            __syncthreads();
            float before = 0.f;
            unsigned n_before = 0;
            for (int w = 0; w < warp; ++w) { before += sm.warp_f[w]; n_before += sm.warp_count[w]; }
            // the border is in front of here at the latest: sums in steps of 2^-24 of themselves, the histogram's own error below 2e-4
            const float goal = weigh ? (float)((double)top_p * S) * 1.001f : (float)top_k;
            if (before + in >= goal && n_before + cnt <= LIST) atomicMin(&sm.bin, tid);
            __syncthreads();
            // (a bin that reaches the goal behind one that holds too much is no answer: sums only grow)
            last_bin = sm.bin;
        } else {
            const double d = -log((double)r.min_p) * 1.4426950408889634 * STEPS;
            last_bin = (int)fmin(ceil(d * 1.00001) + 1.0, (double)(BINS - 1));
        }
        if (last_bin < BINS - 1) {
#pragma unroll 2
            for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                float x[VEC];
                load(i, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if ((int)depth_of(r, x[e]) <= last_bin) {
                        const unsigned p = atomicAdd(cluster.map_shared_rank(&sm.n_list, 0), 1u);
                        if (p < LIST) cluster.map_shared_rank(sm.list, 0)[p] = rank_of(x[e], first + i + e);
                    }
            }
            cluster.sync();
            const int count = (int)*cluster.map_shared_rank(&sm.n_list, 0);
            if (count <= LIST) {
                cluster.sync();                                    // (everybody has read the count)
                if (me != 0) return;
                // sorted along the order
                if (count <= 128) {
                    unsigned long long v = ~0ull;
                    int rank = 0;
                    if (tid < count) {
                        v = sm.list[tid];
                        for (int j = 0; j < count; ++j) rank += sm.list[j] < v;
                    }
                    __syncthreads();
                    if (tid < count) sm.list[rank] = v;
                    __syncthreads();
                } else {
                    int size = 256;
                    while (size < count) size *= 2;
                    for (int i = count + tid; i < size; i += NT) sm.list[i] = ~0ull;
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
                }
                // exact sums along it, a thread for four neighbours: sums up to each of them, and where the front ends
                const int n_k = use_k ? min(count, top_k) : count;
                double w[4], run = 0.0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = tid * 4 + e;
                    w[e] = i < n_k ? weight(r, sm.tab, rank_value(sm.list[i])) : 0.0;
                    if (i < count) sm.list_w[i] = w[e];
                    run += w[e];
                }
                const double in = warp_scan_f64(run, lane);
                if (lane == 31) sm.warp_sum2[warp] = in;
                __syncthreads();
                double upto = in - run, all = 0.0;
                {
                    double before = 0.0;
                    for (int k = 0; k < NW; ++k) {
                        if (k == warp) before = all;
                        all += sm.warp_sum2[k];
                    }
                    upto += before;
                }
                const double theta = use_p ? (double)top_p * (use_k ? all : S) : INFINITY;
                int stay = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = tid * 4 + e;
                    stay += i < n_k && (i == 0 || (upto < theta && w[e] >= r.min_p));
                    upto += w[e];
                }
                stay = __reduce_add_sync(0xffffffffu, stay);
                if (lane == 0) sm.warp_count[warp] = stay;
                __syncthreads();
                int kept = 0;
                for (int k = 0; k < NW; ++k) kept += sm.warp_count[k];
                __syncthreads();
                // The smallest index at which the kept weights in the order of indices exceed uniform times their sum: NW + 1 parts of the range at a time, a warp sums up to each border
                auto sum_to = [&](int index) {                      // a whole warp
                    double t = 0.0;
                    for (int i = lane; i < kept; i += 32)
                        if ((int)(uint32_t)sm.list[i] <= index) t += sm.list_w[i];
                    return warp_sum_f64(t);
                };
                const double W = sum_to(a.vocab), target = (double)uniform * W;
                int lo = -1, hi = a.vocab - 1;                      // the sum up to lo does not exceed the target; up to hi it does, or nothing does
                while (hi - lo > 1) {
                    const int part = (hi - lo - 1) / NW + 1, at = min(hi, lo + (warp + 1) * part);
                    const bool over = at >= hi || sum_to(at) > target;
                    if (lane == 0) sm.warp_count[warp] = over;
                    __syncthreads();
                    int f = 0;
                    while (f < NW && !sm.warp_count[f]) ++f;
                    const int new_hi = f < NW ? min(hi, lo + (f + 1) * part) : hi;
                    lo = min(hi - 1, lo + f * part);
                    hi = new_hi;
                    __syncthreads();
                }
                // the element at hi; with a target that nothing exceeds, the last kept one with weight
                if (warp == 0) {
                    const bool none = !(W > target);
                    int found = -1;
                    if (none) {
                        for (int i = lane; i < kept; i += 32)
                            if (sm.list_w[i] > 0.0) found = max(found, (int)(uint32_t)sm.list[i]);
                        hi = __reduce_max_sync(0xffffffffu, found);
                    }
                    for (int i = lane; i < kept; i += 32)
                        if ((int)(uint32_t)sm.list[i] == hi) {
                            a.tokens[row] = hi;
                            if (a.logprob) a.logprob[row] = (float)log(sm.list_w[i] / W);
                        }
                }
                return;
            }
        }
        cluster.sync();                                            // histograms and count have been read
        if (tid == 0) sm.n_list = 0;
    }

    // ---- fronts too long for the list: what = 0 top-k, 1 top-p
    auto inside = [&](uint32_t k, uint32_t lo, uint32_t hi, int index) {
        return k >= lo && k <= hi && (((unsigned long long)~k << 32) | (unsigned)index) <= r.bound;
    };
    for (int what = 0; what < 2; ++what) {
        if (what == 0 ? !use_k : !use_p) continue;
        double theta = 0.0;               // top-p: the weights that have to be reached
        if (what == 1) {
            if (!have_s || use_k) {
                double s = 0.0;
                for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                    float x[VEC];
                    load(i, x);
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (i + e < n && rank_of(x[e], first + i + e) <= r.bound) s += weight(r, sm.tab, x[e]);
                }
                publish(s);
                cluster.sync();
                S = total();
            }
            theta = (double)top_p * S;
        }
        uint32_t key_lo = 0, key_hi = ~0u;          // keys of the interval that holds the border
        unsigned above = 0;                         // elements in front of it
        double above_w = 0.0;                       // their weights
        int level = 0, width = 0;                   // bins of 2^width keys from level 1 on
        unsigned long long bound = 0;
        for (;;) {
            auto bin = [&](float x, uint32_t k) { return level == 0 ? (int)depth_of(r, x) : (int)((key_hi - k) >> width); };
            sm.hist[tid] = 0;
            __syncthreads();
            for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                float x[VEC];
                load(i, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const uint32_t k = order_key(x[e]);
                    if (i + e < n && inside(k, key_lo, key_hi, first + i + e)) atomicAdd(&sm.hist[bin(x[e], k)], 1u);
                }
            }
            __syncthreads();
            cluster.sync();
            unsigned mine = 0;
            for (int c = 0; c < CL; ++c) mine += cluster.map_shared_rank(sm.hist, c)[tid];
            sm.all[tid] = mine;
            const unsigned in = warp_scan_u32(mine, lane);
            if (lane == 31) sm.warp_count[warp] = in;
            __syncthreads();
            unsigned n_before = above;
            for (int w = 0; w < warp; ++w) n_before += sm.warp_count[w];
            n_before += in - mine;                  // elements in front of this thread's bin
            int at_bin = 0;
            unsigned before = above;
            double before_w = above_w;
            if (what == 0) {
                if (n_before < (unsigned)top_k && (unsigned)top_k <= n_before + mine) { sm.bin = tid; sm.above = n_before; }
                __syncthreads();
                at_bin = sm.bin;
                before = sm.above;
            } else {
                // the bin by halves: exact weights of the bins up to one
                int lo = -1, hi = BINS - 1;         // up to lo they do not reach theta; up to hi they do, or nothing does
                double lo_w = above_w;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    double s = 0.0;
                    for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                        float x[VEC];
                        load(i, x);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            const uint32_t k = order_key(x[e]);
                            if (i + e >= n || !inside(k, key_lo, key_hi, first + i + e)) continue;
                            const int b = bin(x[e], k);
                            if (b > lo && b <= mid) s += weight(r, sm.tab, x[e]);
                        }
                    }
                    publish(s);
                    cluster.sync();
                    const double t = lo_w + total();
                    if (t >= theta) hi = mid;
                    else { lo = mid; lo_w = t; }
                }
                // (where nothing reaches theta, for the last bits of sums taken in another order, the last bin that holds something)
                if (tid == 0) sm.bin = 0;
                __syncthreads();
                if (mine > 0 && tid <= hi) atomicMax(&sm.bin, tid);
                __syncthreads();
                at_bin = sm.bin;
                if (at_bin == tid) sm.above = n_before;
                __syncthreads();
                before = sm.above;
                before_w = lo_w;
                if (at_bin < hi) {                  // the bins behind at_bin are empty: take it out of lo_w again
                    double s = 0.0;
                    for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                        float x[VEC];
                        load(i, x);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            const uint32_t k = order_key(x[e]);
                            if (i + e < n && inside(k, key_lo, key_hi, first + i + e) && bin(x[e], k) < at_bin) s += weight(r, sm.tab, x[e]);
                        }
                    }
                    publish(s);
                    cluster.sync();
                    before_w = above_w + total();
                }
            }
            const unsigned here = sm.all[at_bin];
            // keys of the bin; its elements to the list where they fit
            uint32_t lo = ~0u, hi = 0;
            for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                float x[VEC];
                load(i, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const uint32_t k = order_key(x[e]);
                    if (i + e >= n || !inside(k, key_lo, key_hi, first + i + e) || bin(x[e], k) != at_bin) continue;
                    lo = min(lo, k);
                    hi = max(hi, k);
                    if (here <= LIST) {
                        const unsigned p = atomicAdd(cluster.map_shared_rank(&sm.n_list, 0), 1u);
                        cluster.map_shared_rank(sm.list, 0)[p] = rank_of(x[e], first + i + e);
                    }
                }
            }
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            __syncthreads();
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
                    // sort, then the border by sums along the order
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
                        for (int i = tid; i < (int)here; i += NT) sm.list_w[i] = weight(r, sm.tab, rank_value(sm.list[i]));
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
                    const double m = ceil((theta - before_w) / weight(r, sm.tab, key_value(lo)));
                    take = m >= 1.0 ? (m < (double)here ? (unsigned)m : here) : 1u;       // (weights of nothing: one of them)
                }
                auto same = [&](int i, float (&x)[VEC]) {        // of a lane's elements as bits
                    load(i, x);
                    unsigned bits = 0;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) bits |= (unsigned)(i + e < n && order_key(x[e]) == lo && rank_of(x[e], first + i + e) <= r.bound) << e;
                    return bits;
                };
                unsigned c = 0;
                float x[VEC];
                for (int i = w0 + lane * VEC; i < w1; i += STRIDE) c += __popc(same(i, x));
                c = __reduce_add_sync(0xffffffffu, c);
                __syncthreads();
                if (lane == 0) sm.warp_count[warp] = c;
                __syncthreads();
                if (tid < CL) {
                    unsigned t = 0;
                    for (int w = 0; w < NW; ++w) t += sm.warp_count[w];
                    cluster.map_shared_rank(sm.count, tid)[me] = t;
                }
                cluster.sync();
                unsigned run = 0;
                for (int k = 0; k < me; ++k) run += sm.count[k];
                for (int w = 0; w < warp; ++w) run += sm.warp_count[w];
                if (run < take && take <= run + sm.warp_count[warp]) {
                    for (int i0 = w0; i0 < w1; i0 += STRIDE) {
                        const int i = i0 + lane * VEC;
                        const unsigned bits = i < w1 ? same(i, x) : 0u;
                        const unsigned upto = warp_scan_u32(__popc(bits), lane);
                        unsigned left = take - run - (upto - __popc(bits));          // the how manieth of this lane's
                        if (left >= 1 && left <= (unsigned)__popc(bits))
                            for (int e = 0; e < VEC; ++e)
                                if (((bits >> e) & 1) && --left == 0)
                                    for (int k = 0; k < CL; ++k) *cluster.map_shared_rank(&sm.answer, k) = rank_of(key_value(lo), first + i + e);
                        run += __shfl_sync(0xffffffffu, upto, 31);
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
    auto kept_weight = [&](float x, int index) {
        if (rank_of(x, index) > r.bound) return 0.0;
        const double w = weight(r, sm.tab, x);
        return w >= r.min_p ? w : 0.0;
    };
    double s = 0.0;
#pragma unroll 2
    for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
        float x[VEC];
        load(i, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += kept_weight(x[e], first + i + e);
    }
    publish(s);
    cluster.sync();
    const double W = total(), target = (double)uniform * W;
    double run = 0.0;
    for (int c = 0; c < me; ++c) run += sm.sum[flip][c];
    // a block has the token if the target lies in its share; the last one with weight takes what rounding leaves behind it
    bool last = true;
    for (int c = me + 1; c < CL; ++c) last = last && sm.sum[flip][c] == 0.0;
    const double mine = sm.sum[flip][me];
    if (!(mine > 0.0 && target >= run && (target < run + mine || last))) return;
    // the first warp whose weights exceed it, or the last one with weight
    int owner = -1;
    for (int w = 0; w < NW; ++w) {
        if (sm.warp_sum[w] == 0.0) continue;
        if (owner >= 0) run += sm.warp_sum[owner];
        owner = w;
        if (run + sm.warp_sum[w] > target) break;
    }
    if (warp != owner) return;
    int token = -1;
    double w_token = 0.0;
    for (int i0 = w0; i0 < w1; i0 += STRIDE) {
        const int i = i0 + lane * VEC;
        float x[VEC];
        double w[VEC], sum = 0.0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = 0.0;
        if (i < w1) {
            load(i, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                w[e] = kept_weight(x[e], first + i + e);
                sum += w[e];
            }
        }
        const double in = warp_scan_f64(sum, lane);
        const uint32_t hit = __ballot_sync(0xffffffffu, sum > 0.0 && run + in > target), some = __ballot_sync(0xffffffffu, sum > 0.0);
        if (some) {
            const int src = hit ? __ffs(hit) - 1 : 31 - __clz(some);
            double upto = run + in - sum;
            int at = -1;
            double w_at = 0.0;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (w[e] > 0.0 && !(at >= 0 && upto > target)) { at = e; w_at = w[e]; }
                upto += w[e];
            }
            token = __shfl_sync(0xffffffffu, first + i + at, src);
            w_token = __shfl_sync(0xffffffffu, w_at, src);
        }
        if (hit) break;
        run += __shfl_sync(0xffffffffu, in, 31);
    }
    if (lane == 0) {
        a.tokens[row] = token;
        if (a.logprob) a.logprob[row] = (float)log(w_token / W);
    }
}

template <typename T>
int run(SampleArgs a, cudaStream_t s) {
    constexpr int STRIDE = 32 * Raw<T>::VEC;
    int cl = 1;
    while (cl < MAX_CL && a.vocab > cl * 4096) cl *= 2;
    a.chunk = ((a.vocab + cl - 1) / cl + STRIDE - 1) / STRIDE * STRIDE;
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
    if (n_rows < 0 || n_rows > (1 << 27) || vocab < 1 || vocab > MAX_VOCAB || row_stride < 0 || row_stride > ((int64_t)1 << 40) || !sampling) return ESP_E_ARG;
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
