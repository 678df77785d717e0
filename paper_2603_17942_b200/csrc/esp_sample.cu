// Sampling from rows of logits: temperature, top-k, top-p and min-p, from one given random number a row.
//
// The order: larger logits first, of equal ones the lower index.  top-k, top-p and min-p each keep a front of it.  Weights are exp((x - M) / temperature) in 64 bits, M the row's
// largest, and their sums are in 64 bits in a fixed order wherever a sum decides: the front of top-p ends where a sum meets top_p times another, and the draw where one exceeds
// uniform times another.  The token is found along the indices, not along the order, so that nothing has to be sorted but what the limits ask for.
//
//   scan   a block for each slice of 8192 logits of a row, which it holds in its registers and reads once: the slice's largest element, the sums of its weights by stretches of 1024
//          (for top-p and for rows without limits), and a list of its largest elements, about 110, with the value below which it leaves things out.  How many weights it has to
//          work out is what bounds it where sums are asked for (us, 272 fp32 rows of 128256, 20 us to read: greedy 28, temperature alone 54, min-p 62).
//   list   a block for each row: the slices' largest give M, and the sums scaled to it the row's S.  What the limits keep lies nearly always within the lists: histograms say how far,
//          those elements are sorted, their exact sums cut, and the draw is among them.  Rows without limits draw by stretches: the one the target lies in, then its element.
//   rest   clusters of up to eight blocks for the rows that the lists do not settle.
//          Long fronts of top-p (thousands of elements): a histogram of the weights over the whole row says in which bin of 1/25 of a logit the front ends; then sums of what lies in
//          front of the bin, with that bin's elements as lists; the end by exact sums along them; the draw by stretches.  About 30 us for one row of 128256.
//          Everything else (long fronts of top-k, thousands of equal logits, infinite logits): a value that the front does not reach below, or, where too much lies above it, the
//          front's last element by histograms that close in on it; then the draw by stretches.
// Sorting whole rows is what this avoids: with the row in a cluster's shared memory and every limit's end found there, the same 272 rows took 200 to 480 us instead of 54 to 157.
#include <cooperative_groups.h>
#include <math.h>

#include "esp_paged.cuh"

namespace cg = cooperative_groups;

namespace esp {

namespace {

using paged::warp_scan_u32;

constexpr int NT = 512, NW = NT / 32;
constexpr int BINS = SAMPLE_BINS;         // of a histogram, a thread for each
static_assert(BINS == NT, "");
constexpr float STEPS = 24.f;             // fine bins of an octave of weights: 21 octaves
constexpr int FINE = 256, COARSE = 8;     // wide bins: that many fine ones, then as wide as eight of them: 95 octaves
constexpr int MAX_CL = 8;                 // blocks of a cluster at most
constexpr int LIST = 2048;                // elements that are sorted at most
constexpr int SMEM_ROW = 64 * 1024;       // bytes of a row that a block keeps at most: two blocks an SM (us, 64 fp32 rows of 128256, top-k 2500: kept 141, read anew 175)
constexpr int TAB = 256;                  // 2^(j / TAB)
constexpr float UNIT = SAMPLE_UNIT, GRID = 25.f;   // a histogram of weights counts in 1 / UNIT (or less: sample_unit) of what a bin's upper end weighs, bins are 1 / GRID of a logit
static_assert(sample_unit(SAMPLE_MAX_SLICES * SAMPLE_CAP) == SAMPLE_UNIT, "all lists' elements may be in one bin");
constexpr int MAX_VOCAB = SAMPLE_MAX_SLICES * SAMPLE_SLICE;      // 2^21
constexpr int WANT = 110;                 // elements of a slice that go to its list, more or less

// 2^(j / TAB), as the compiler works it out: the series of exp(j ln 2 / TAB)
struct PowTable {
    double v[TAB];
    constexpr PowTable() : v() {
        for (int j = 0; j < TAB; ++j) {
            const double x = j * (0.6931471805599453 / TAB);
            double sum = 0.0;
            for (int k = 24; k > 0; --k) sum = (sum + 1.0) * x / k;
            v[j] = sum + 1.0;
        }
    }
};
__device__ const PowTable POW_TABLE;

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
    double sum[2][MAX_CL];                // a sum of each block
    unsigned count[MAX_CL];
    uint32_t lo[MAX_CL], hi[MAX_CL];      // smallest and largest key of an interval in each block
    uint32_t hist[BINS];
    uint32_t all[BINS];                   // the cluster's
    unsigned long long list[LIST];        // the first block's
    double list_w[LIST];
    uint32_t n_list;
    uint32_t n_of[MAX_CL];                // elements of each block's list
    double warp_sum[NW], warp_sum2[NW], kept_sum;
    int kept;
    float warp_f[NW];
    unsigned warp_count[NW];
    uint32_t warp_lo[NW], warp_hi[NW];
    unsigned long long answer;
    int verdict;
    int bin, end_bin;
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

// exp((x - M) / temperature), M finite: 2^n * 2^(j / 256) from a table * a polynomial of degree 3 on what is left, |d| <= 1/512 octave: (ln 2 / 512)^4 / 24 = 1.4e-13 of the
// weight.  Weights below 2^-120 of the largest count as nothing.  Passes over whole rows are bound by how many instructions this takes.
__device__ __forceinline__ double weight(const Row& r, const double* tab, float x) {
    constexpr double C1 = 0.6931471805599453 / TAB, C2 = C1 * C1 / 2, C3 = C1 * C1 * C1 / 6, MAGIC = 6755399441055744.0;      // 1.5 * 2^52: the sum's last bits are the whole number
    const double diff = (double)x - r.Md, u = fma(diff, r.A, MAGIC), d = fma(diff, r.A, MAGIC - u);
    const int n = __double2loint(u);
    const double v = tab[n & (TAB - 1)], p = fma(v * d, fma(d, fma(d, C3, C2), C1), v);
    const double w = __hiloint2double(__double2hiint(p) + ((n & ~(TAB - 1)) << 12), __double2loint(p));
    return u > MAGIC - 120.0 * TAB ? w : 0.0;
}
// Fine bins from the largest logit down; BINS - 1: somewhere behind.
__device__ __forceinline__ float depth_of(const Row& r, float x) { return x == r.M ? 0.f : fminf((r.M - x) * r.steps, (float)(BINS - 1)); }

// The same with a range four times as far
__device__ __forceinline__ int wide_bin(const Row& r, float x) {
    const float d = x == r.M ? 0.f : fminf((r.M - x) * r.steps, (float)(BINS * COARSE));
    return d < (float)FINE ? (int)d : min(FINE + (int)((d - (float)FINE) * (1.f / COARSE)), BINS - 1);
}
__device__ __forceinline__ float wide_end(int bin) { return bin < FINE ? (float)(bin + 1) : (float)(FINE + (bin + 1 - FINE) * COARSE); }

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

// Sorts the block's list along the order and puts the elements' weights beside it.  Called by all threads.
template <typename T>
__device__ __forceinline__ void sort_list(const Row& r, Shared& sm, int vocab, int count) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __syncthreads();
    if (count <= 128) {
        // each element counts the ones in front of it
        unsigned long long v = ~0ull;
        int rank = 0;
        if (tid < count) {
            v = sm.list[tid];
#pragma unroll 4
            for (int j = 0; j < count; ++j) rank += sm.list[j] < v;
        }
        __syncthreads();
        if (tid < count) {
            sm.list[rank] = v;
            sm.list_w[rank] = weight(r, sm.tab, rank_value(v));
        }
        __syncthreads();
        return;
    }
    // by bins of (key, index), then each element counts the ones in front of it in its bin.  bf16 has few different keys in a list, with bits that are the same in all: without
    // these the numbers that are cut into bins lie dense, by the indices (several hundred equal logits in one bin took 20 us to be put in order)
    constexpr int SAME = sizeof(T) == 2 ? 16 : 0;
    constexpr int PER = LIST / NT;
    unsigned long long v[PER];
    uint32_t lo = ~0u, hi = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e)
        if (e * NT + tid < count) {
            v[e] = sm.list[e * NT + tid];
            const uint32_t k = (uint32_t)(v[e] >> 32);
            lo = min(lo, k);
            hi = max(hi, k);
        }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) { sm.warp_lo[warp] = lo; sm.warp_hi[warp] = hi; }
    sm.hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) { lo = min(lo, sm.warp_lo[w]); hi = max(hi, sm.warp_hi[w]); }
    // values far from each other: by their distance from the largest instead, for keys would leave most bins to what is next to zero; what has no weight is last, in any order
    const bool wide = hi - lo > 2u << 23;
    const float top = key_value(~lo), scale = (BINS - 2) / fminf(top - key_value(~hi), (float)(121.0 * TAB / r.A));
    lo >>= SAME;
    const int bits = 32 - __clz(vocab - 1), width = max(0, bits + 32 - __clz((hi >> SAME) - lo) - 9);
    static_assert(BINS == 1 << 9, "");
    int bin[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        bin[e] = -1;
        if (e * NT + tid < count) {
            if (!wide) bin[e] = (int)((((unsigned long long)((uint32_t)(v[e] >> 32) >> SAME) - lo) << bits | (uint32_t)v[e]) >> width);
            else {
                const float x = rank_value(v[e]);
                bin[e] = weight(r, sm.tab, x) == 0.0 ? BINS - 1 : min((int)((top - x) * scale), BINS - 2);
            }
            atomicAdd(&sm.hist[bin[e]], 1u);
        }
    }
    __syncthreads();
    const unsigned mine = sm.hist[tid], in = warp_scan_u32(mine, lane), most = __reduce_max_sync(0xffffffffu, wide && tid == BINS - 1 ? 0u : mine);
    if (lane == 31) { sm.warp_count[warp] = in; sm.warp_hi[warp] = most; }
    __syncthreads();
    unsigned begin = in - mine, largest = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        begin += w < warp ? sm.warp_count[w] : 0u;
        largest = max(largest, sm.warp_hi[w]);
    }
    sm.all[tid] = begin;
    sm.hist[tid] = begin;
    __syncthreads();
    if (largest <= 512) {
        int rank[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (bin[e] >= 0) {
                rank[e] = atomicAdd(&sm.hist[bin[e]], 1u);
                sm.list[rank[e]] = v[e];
            }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (bin[e] >= 0 && !(wide && bin[e] == BINS - 1)) {
                const int j0 = sm.all[bin[e]], j1 = sm.hist[bin[e]];
                int at = j0;
#pragma unroll 4
                for (int j = j0; j < j1; ++j) at += sm.list[j] < v[e];
                rank[e] = at;
            }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (bin[e] >= 0) {
                sm.list[rank[e]] = v[e];
                sm.list_w[rank[e]] = weight(r, sm.tab, rank_value(v[e]));
            }
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
        for (int i = tid; i < count; i += NT) sm.list_w[i] = weight(r, sm.tab, rank_value(sm.list[i]));
    }
    __syncthreads();
}

// What a block does with a list of `count` elements, the first ones of the order: sorts it, cuts it and draws.  S: the weights of the whole row that top_p goes by (below 0: those of
// the first top_k).  whole: what is not in the list is not kept.  false: top_p reaches beyond the list.
template <typename T>
__device__ __forceinline__ bool from_list(const Row& r, Shared& sm, const SampleArgs& a, int row, int count, int top_k, float top_p, double S, float uniform, bool whole) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    sort_list<T>(r, sm, a.vocab, count);

    // ---- exact sums along it, four neighbours a lane, and where the front ends
    const int n_k = min(count, top_k);
    const bool one_warp = n_k <= 128;
    if (!one_warp || warp == 0) {
        double w[4], run = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = tid * 4 + e;
            w[e] = i < n_k ? sm.list_w[i] : 0.0;
            run += w[e];
        }
        const double in = warp_scan_f64(run, lane);
        double upto = in - run, all = __shfl_sync(0xffffffffu, in, 31);
        if (!one_warp) {
            if (lane == 31) sm.warp_sum2[warp] = in;
            __syncthreads();
            all = 0.0;
            double before = 0.0;
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                if (k == warp) before = all;
                all += sm.warp_sum2[k];
            }
            upto += before;
        }
        const double theta = top_p < 1.f ? (double)top_p * (S < 0.0 ? all : S) : INFINITY;
        if (tid == 0) sm.verdict = !whole && S >= 0.0 && top_p < 1.f && all < theta;
        int stay = 0;
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = tid * 4 + e;
            const bool in_front = i < n_k && (i == 0 || (upto < theta && w[e] >= r.min_p));
            stay += in_front;
            upto += w[e];
            if (in_front) sum += w[e];
        }
        stay = __reduce_add_sync(0xffffffffu, stay);
        sum = warp_sum_f64(sum);
        if (one_warp) {
            if (lane == 0) { sm.kept = stay; sm.kept_sum = sum; }
        } else if (lane == 0) { sm.warp_count[warp] = stay; sm.warp_sum[warp] = sum; }
    }
    __syncthreads();
    if (sm.verdict) return false;
    int kept = 0;
    double W = 0.0;
    if (one_warp) {
        kept = sm.kept;
        W = sm.kept_sum;
    } else {
#pragma unroll
        for (int k = 0; k < NW; ++k) { kept += sm.warp_count[k]; W += sm.warp_sum[k]; }
    }
    const double target = (double)uniform * W;

    // ---- the smallest index at which the kept weights in the order of indices exceed the target; with a target that nothing exceeds, the last kept one with weight
    if (kept <= 128) {
        // each element adds up those that its index has in front of it.  (0xffffffff: no candidate)
        if (warp >= 4) return true;
        if (warp == 0 || warp * 32 < kept) {
            const int mine = tid < kept ? (int)(uint32_t)sm.list[tid] : -1;
            double upto = 0.0;
#pragma unroll 4
            for (int j = 0; j < kept; ++j)
                if ((int)(uint32_t)sm.list[j] <= mine) upto += sm.list_w[j];
            const bool has = tid < kept && sm.list_w[tid] > 0.0;
            const unsigned over = __reduce_min_sync(0xffffffffu, has && upto > target ? (unsigned)mine : ~0u);
            const unsigned last = __reduce_max_sync(0xffffffffu, has ? (unsigned)mine + 1u : 0u);
            if (lane == 0) { sm.all[warp] = over; sm.all[4 + warp] = last; }
        } else if (lane == 0) { sm.all[warp] = ~0u; sm.all[4 + warp] = 0u; }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        unsigned over = ~0u, last = 0u;
#pragma unroll
        for (int k = 0; k < 4; ++k) { over = min(over, sm.all[k]); last = max(last, sm.all[4 + k]); }
        const unsigned token = over != ~0u ? over : last - 1u;
        if (tid < kept && (uint32_t)sm.list[tid] == token) {
            a.tokens[row] = (int)token;
            if (a.logprob) a.logprob[row] = (float)log(sm.list_w[tid] / W);
        }
        return true;
    }
    // the range of indices in NW parts at a time: a warp sums up to each border
    int lo = -1, hi = a.vocab - 1;                                  // the sum up to lo does not exceed the target; up to hi it does, or nothing does
    while (hi - lo > 1) {
        const int part = (hi - lo - 1) / NW + 1, at = min(hi, lo + (warp + 1) * part);
        double t = 0.0;
        for (int i = lane; i < kept; i += 32)
            if ((int)(uint32_t)sm.list[i] <= at) t += sm.list_w[i];
        const bool over = at >= hi || warp_sum_f64(t) > target;
        __syncthreads();
        if (lane == 0) sm.warp_count[warp] = over;
        __syncthreads();
        const uint32_t overs = __ballot_sync(0xffffffffu, lane < NW && sm.warp_count[lane & (NW - 1)]);
        const int f = __ffs(overs) - 1;                             // (the last border is always over)
        const int new_hi = min(hi, lo + (f + 1) * part);
        lo = min(hi - 1, lo + f * part);
        hi = new_hi;
    }
    if (warp == 0) {
        if (!(W > target)) {
            unsigned last = 0;
            for (int i = lane; i < kept; i += 32)
                if (sm.list_w[i] > 0.0) last = max(last, (uint32_t)sm.list[i]);
            hi = (int)__reduce_max_sync(0xffffffffu, last);
        }
        for (int i = lane; i < kept; i += 32)
            if ((int)(uint32_t)sm.list[i] == hi) {
                a.tokens[row] = hi;
                if (a.logprob) a.logprob[row] = (float)log(sm.list_w[i] / W);
            }
    }
    return true;
}

// A row's settings.
struct Limits {
    float temperature, uniform, top_p, min_p;
    int top_k;
    bool bad, use_k, use_p, use_m, one;       // one: only the first element stays
};
__device__ __forceinline__ Limits limits_of(const SampleArgs& a, int row) {
    Limits l;
    l.temperature = a.temperature ? __ldg(a.temperature + row) : 1.f;
    l.uniform = __ldg(a.uniform + row);
    l.top_k = a.top_k ? __ldg(a.top_k + row) : 0;
    l.top_p = a.top_p ? __ldg(a.top_p + row) : 1.f;
    l.min_p = a.min_p ? __ldg(a.min_p + row) : 0.f;
    l.bad = !(l.temperature >= 0.f) || isinf(l.temperature) || !(l.uniform >= 0.f) || l.top_p != l.top_p || l.min_p != l.min_p;
    l.use_k = l.top_k >= 1 && l.top_k < a.vocab;
    l.use_p = l.top_p < 1.f;
    l.use_m = l.min_p > 0.f;
    l.one = l.temperature == 0.f || l.top_k == 1 || l.top_p <= 0.f;
    return l;
}
__device__ __forceinline__ void set_row(Row& r, const Limits& l, float M) {
    const double inv_t = 1.0 / (double)l.temperature;
    r.M = M;
    r.Md = (double)M;
    r.A = inv_t * (TAB * 1.4426950408889634);
    r.steps = (float)fmin(inv_t * ((double)STEPS * 1.4426950408889634), 3e38);
    r.bound = ~0ull;
    r.min_p = fmin((double)l.min_p, 1.0);
}

constexpr int SCAN_THREADS = 256, SCAN_WARPS = SCAN_THREADS / 32, SLICE = SAMPLE_SLICE, CAP = SAMPLE_CAP, STRETCH = SLICE / SCAN_WARPS;
constexpr int PER_STRETCH = SAMPLE_MAX_SLICES * SCAN_WARPS / NT;      // stretches of a thread of the second pass

// The token, given the kept weights w of PER_STRETCH stretches of each thread in their order and their sum W: the stretch in which the target lies, or the last one with
// weight, then its element.  All threads of a block.
template <typename T>
__device__ __forceinline__ void draw_from(const Row& r, Shared& sm, const SampleArgs& a, int row, const double (&w)[PER_STRETCH], double W, double target) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int NONE = 1 << 30, E = STRETCH / NT;
    double run = 0.0;
#pragma unroll
    for (int e = 0; e < PER_STRETCH; ++e) run += w[e];
    const double in = warp_scan_f64(run, lane);
    __syncthreads();
    if (lane == 31) sm.warp_sum[warp] = in;
    if (tid == 0) { sm.bin = NONE; sm.end_bin = -1; }
    __syncthreads();
    double upto = in - run;
#pragma unroll
    for (int k = 0; k < NW; ++k) upto += k < warp ? sm.warp_sum[k] : 0.0;
    int found = NONE, last = -1;
    double found_front = 0.0, last_front = 0.0;
#pragma unroll
    for (int e = 0; e < PER_STRETCH; ++e) {
        if (w[e] > 0.0) {
            last = tid * PER_STRETCH + e;
            last_front = upto;
            if (found == NONE && upto + w[e] > target) { found = last; found_front = upto; }
        }
        upto += w[e];
    }
    const int f = __reduce_min_sync(0xffffffffu, found), z = __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) { atomicMin(&sm.bin, f); atomicMax(&sm.end_bin, z); }
    __syncthreads();
    const bool none = sm.bin == NONE;
    const int at = none ? sm.end_bin : sm.bin;
    if (none ? last == at : found == at) sm.kept_sum = none ? last_front : found_front;
    __syncthreads();
    // neighbours a thread
    const T* logits = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride;
    const int i0 = at * STRETCH + tid * E;
    double v[E], sum = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = i0 + e < a.vocab ? number(to_f32(logits[i0 + e])) : -INFINITY;
        v[e] = rank_of(x, i0 + e) <= r.bound ? weight(r, sm.tab, x) : 0.0;
        sum += v[e];
    }
    const double scan = warp_scan_f64(sum, lane);
    if (lane == 31) sm.warp_sum2[warp] = scan;
    if (tid == 0) { sm.bin = NONE; sm.end_bin = -1; }
    __syncthreads();
    double here = sm.kept_sum + scan - sum;
#pragma unroll
    for (int k = 0; k < NW; ++k) here += k < warp ? sm.warp_sum2[k] : 0.0;
    int hit = NONE, some = -1;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        here += v[e];
        if (v[e] > 0.0) {
            some = tid * E + e;
            if (hit == NONE && here > target) hit = some;
        }
    }
    const int h = __reduce_min_sync(0xffffffffu, hit), y = __reduce_max_sync(0xffffffffu, some);
    if (lane == 0) { atomicMin(&sm.bin, h); atomicMax(&sm.end_bin, y); }
    __syncthreads();
    const int token = sm.bin < NONE ? sm.bin : sm.end_bin;
    if (token / E == tid) {
        a.tokens[row] = at * STRETCH + token;
        if (a.logprob) a.logprob[row] = (float)log((token % E ? v[E - 1] : v[0]) / W);
    }
}

// Bins on a grid that all rows share, 1/25 of a logit each: bin k holds the logits from k / GRID on.
__device__ __forceinline__ int grid_bin(float x) { return __float2int_rd(x * GRID); }
// What an element adds to its bin of weights, in 1 / unit of the weight of the bin's upper end; per: log2 e / (GRID temperature).
__device__ __forceinline__ unsigned grid_weight(float x, int k, float per, float unit) { return __float2uint_rn(unit * exp2f((x * GRID - (float)(k + 1)) * per)); }

// A slice of n logits, VEC of them to a lane at i0, i0 + 32 VEC, ...; -infinity behind its end.
template <typename T>
__device__ __forceinline__ void load_slice(const T* x0, int n, int i0, uint4 (&raw)[SLICE / SCAN_THREADS / Raw<T>::VEC]) {
    constexpr int VEC = Raw<T>::VEC, PER = SLICE / SCAN_THREADS / VEC;
    const bool aligned = reinterpret_cast<uintptr_t>(x0) % 16 == 0;
    if (n == SLICE && aligned) {
#pragma unroll
        for (int j = 0; j < PER; ++j) raw[j] = __ldg(reinterpret_cast<const uint4*>(x0 + i0 + j * 32 * VEC));
        return;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int i = i0 + j * 32 * VEC;
        if (aligned && i + VEC <= n) raw[j] = __ldg(reinterpret_cast<const uint4*>(x0 + i));
        else {
            float x[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = i + e < n ? to_f32(x0[i + e]) : -INFINITY;
            raw[j] = Raw<T>::pack(x);
        }
    }
}
// The elements that `bits` marks of SCAN_THREADS threads' into a list of CAP, in the order of warps and lanes; how many there are.  All threads of the block (s_count: their part's).
template <typename T>
__device__ __forceinline__ unsigned put_bits(const uint4 (&raw)[SLICE / SCAN_THREADS / Raw<T>::VEC], uint32_t bits, unsigned* s_count, unsigned long long* list, int index0) {
    constexpr int VEC = Raw<T>::VEC, PER = SLICE / SCAN_THREADS / VEC;
    const int lane = threadIdx.x & 31, warp = (threadIdx.x % SCAN_THREADS) >> 5;
    const unsigned upto = warp_scan_u32(__popc(bits), lane);
    __syncthreads();
    if (lane == 31) s_count[warp] = upto;
    __syncthreads();
    unsigned at = upto - __popc(bits), all = 0;
#pragma unroll
    for (int w = 0; w < SCAN_WARPS; ++w) {
        at += w < warp ? s_count[w] : 0u;
        all += s_count[w];
    }
    if (all <= CAP && __any_sync(0xffffffffu, bits)) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            float x[VEC];
            Raw<T>::unpack(raw[j], x);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if ((bits >> (j * VEC + e)) & 1) list[at++] = rank_of(x[e], index0 + j * 32 * VEC + e);
        }
    }
    return all;
}

// A long front of top-p, first step: a histogram of the row's weights.  The cluster's blocks take the row's slices, half a block for each.  Gives the bin in which the front ends (or its neighbour, at a border
// of bins); false: it is not known, or has more elements than can be sorted (each adds one unit at most, so the bin's sum tells).
template <typename T>
__device__ __forceinline__ bool front_bins(const Row& r, Shared& sm, const SampleArgs& a, const SampleRest& known, float top_p, int& bin, int me, int CL) {
    constexpr int VEC = Raw<T>::VEC, PER = SLICE / SCAN_THREADS / VEC;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, base = grid_bin(known.M);
    const float per = r.steps * (1.f / (STEPS * GRID));
    for (int s0 = 2 * me; s0 < a.slices; s0 += 2 * CL) {
        const int first = (s0 + tid / SCAN_THREADS) * SLICE, n = max(0, min(SLICE, a.vocab - first)), i0 = warp % SCAN_WARPS * STRETCH + lane * VEC;
        uint4 raw[PER];
        load_slice<T>(reinterpret_cast<const T*>(a.logits) + (long long)known.row * a.row_stride + first, n, i0, raw);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            float x[VEC];
            Raw<T>::unpack(raw[j], x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int k = grid_bin(x[e]);
                if ((uint32_t)base - (uint32_t)k < BINS && x[e] == x[e]) atomicAdd(&sm.hist[base - k], grid_weight(x[e], k, per, a.unit));
            }
        }
    }
    cluster.sync();
    uint32_t part[MAX_CL];
#pragma unroll
    for (int c = 0; c < MAX_CL; ++c) part[c] = c < CL ? cluster.map_shared_rank(sm.hist, c)[tid] : 0u;
    unsigned long long mine = 0;
#pragma unroll
    for (int c = 0; c < MAX_CL; ++c) mine += part[c];
    // sums along the bins, by what each one's upper end weighs
    const float v = (float)mine * a.per_unit * exp2f(((float)(base - tid + 1) - known.M * GRID) * per);
    float in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float y = __shfl_up_sync(0xffffffffu, in, o);
        if (lane >= o) in += y;
    }
    if (lane == 31) sm.warp_f[warp] = in;
    if (tid == 0) sm.bin = BINS;
    __syncthreads();
    float before = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) before += w < warp ? sm.warp_f[w] : 0.f;
    if (before + in >= (float)((double)top_p * known.S)) atomicMin(&sm.bin, tid);
    __syncthreads();
    bin = base - sm.bin;
    const bool found = sm.bin < BINS && !__syncthreads_or(tid == sm.bin && mine > (unsigned long long)LIST * (unsigned)a.unit);
    cluster.sync();                       // (the histograms have been read)
    return found;
}

// A long front of top-p, second step: what lies in front of the bin is added up, by stretches, and its elements go to the slices' lists.
template <typename T>
__device__ __forceinline__ void front_slices(const Row& r, Shared& sm, const SampleArgs& a, const SampleRest& known, int bin, int me, int CL) {
    constexpr int VEC = Raw<T>::VEC, PER = SLICE / SCAN_THREADS / VEC;
    const int tid = threadIdx.x, lane = tid & 31, half = tid / SCAN_THREADS, warp = (tid % SCAN_THREADS) >> 5;
    for (int s0 = 2 * me; s0 < a.slices; s0 += 2 * CL) {                 // the same trips in every thread
        const int slice = s0 + half, first = slice * SLICE, n = max(0, min(SLICE, a.vocab - first)), i0 = warp * STRETCH + lane * VEC;
        uint4 raw[PER];
        load_slice<T>(reinterpret_cast<const T*>(a.logits) + (long long)known.row * a.row_stride + first, n, i0, raw);
        double s = 0.0;
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            float x[VEC];
            Raw<T>::unpack(raw[j], x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                x[e] = number(x[e]);
                const int k = grid_bin(x[e]);
                const double w = weight(r, sm.tab, x[e]);
                s += k > bin ? w : 0.0;
                bits |= (uint32_t)(k == bin && i0 + j * 32 * VEC + e < n) << (j * VEC + e);
            }
            raw[j] = Raw<T>::pack(x);
        }
        s = warp_sum_f64(s);
        const unsigned listed = put_bits<T>(raw, bits, sm.warp_count + half * SCAN_WARPS, a.entries + ((size_t)known.row * a.slices + slice) * CAP, first + i0);
        if (slice < a.slices) {
            SampleSlice* out = a.slice + (size_t)known.row * a.slices + slice;
            if (lane == 0) out->stretch[warp] = s;
            if (tid % SCAN_THREADS == 0) {
                out->n = listed <= CAP ? (int)listed : 0;
                out->cut = listed <= CAP ? 0.f : INFINITY;
            }
        }
    }
}

// Third step, by one block: the end of the front is found among the listed elements, the draw is by stretches.  -1: it ends in a bin of larger logits,
// 1: of smaller ones, 2: there are too many elements.
template <typename T>
__device__ __forceinline__ int from_front(Row& r, Shared& sm, const SampleArgs& a, const SampleRest& known, float top_p, float uniform) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const SampleSlice* slice = a.slice + (size_t)known.row * a.slices;
    const unsigned long long* entries = a.entries + (size_t)known.row * a.slices * CAP;
    double w[PER_STRETCH], run = 0.0;
#pragma unroll
    for (int e = 0; e < PER_STRETCH; ++e) {
        const int i = tid * PER_STRETCH + e;
        w[e] = i / SCAN_WARPS < a.slices ? __ldcg(&slice[i / SCAN_WARPS].stretch[i % SCAN_WARPS]) : 0.0;
        run += w[e];
    }
    if (tid < a.slices) sm.all[tid] = __ldcg(&slice[tid].n);
    const bool over = __syncthreads_or(tid < a.slices && __ldcg(&slice[tid].cut) == INFINITY);
    if (over) return 2;
    for (int i = tid; i < a.slices * CAP; i += NT)
        if (i % CAP < (int)sm.all[i / CAP]) {
            const unsigned at = atomicAdd(&sm.n_list, 1u);
            if (at < LIST) sm.list[at] = __ldcg(entries + i);
        }
    const double all_in = warp_scan_f64(run, lane);
    if (lane == 31) sm.warp_sum[warp] = all_in;
    __syncthreads();
    const int count = (int)sm.n_list;
    double before = 0.0;
#pragma unroll
    for (int k = 0; k < NW; ++k) before += sm.warp_sum[k];
    const double theta = (double)top_p * known.S;
    if (before >= theta) return -1;
    if (count < 1) return 1;
    if (count > LIST) return 2;
    // the first element at which the sums along the order reach theta, four neighbours a thread
    sort_list<T>(r, sm, a.vocab, count);
    constexpr int PER = LIST / NT, NONE = 1 << 30;
    double v[PER], part = 0.0;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        v[e] = tid * PER + e < count ? sm.list_w[tid * PER + e] : 0.0;
        part += v[e];
    }
    const double in = warp_scan_f64(part, lane);
    if (lane == 31) sm.warp_sum2[warp] = in;
    if (tid == 0) sm.bin = NONE;
    __syncthreads();
    double upto = before + in - part, W = 0.0;
#pragma unroll
    for (int k = 0; k < NW; ++k) upto += k < warp ? sm.warp_sum2[k] : 0.0;
    int end = NONE;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        upto += v[e];
        if (end == NONE && tid * PER + e < count && upto >= theta) { end = tid * PER + e; W = upto; }
    }
    const int first = __reduce_min_sync(0xffffffffu, end);
    if (lane == 0) atomicMin(&sm.bin, first);
    __syncthreads();
    if (sm.bin == NONE) return 1;
    if (end == sm.bin) { sm.kept_sum = W; sm.answer = sm.list[end]; }
    __syncthreads();
    W = sm.kept_sum;
    r.bound = sm.answer;
    // what of the lists is kept, by stretches (the sorted list is done with: its place has the sums)
    double* kept = reinterpret_cast<double*>(sm.list);
    for (int s = warp; s < a.slices; s += NW) {
        const int n = (int)__ldcg(&slice[s].n);
        double sum[SCAN_WARPS];
#pragma unroll
        for (int e = 0; e < SCAN_WARPS; ++e) sum[e] = 0.0;
        for (int i = lane; i < n; i += 32) {
            const unsigned long long x = __ldcg(entries + (size_t)s * CAP + i);
            const double y = x <= r.bound ? weight(r, sm.tab, rank_value(x)) : 0.0;
            const int at = ((int)(uint32_t)x - s * SLICE) / STRETCH;
#pragma unroll
            for (int e = 0; e < SCAN_WARPS; ++e) sum[e] += e == at ? y : 0.0;
        }
#pragma unroll
        for (int e = 0; e < SCAN_WARPS; ++e) {
            const double y = warp_sum_f64(sum[e]);
            if (lane == 0) kept[s * SCAN_WARPS + e] = y;
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PER_STRETCH; ++e) {
        const int i = tid * PER_STRETCH + e;
        if (i / SCAN_WARPS < a.slices) w[e] += kept[i];
    }
    draw_from<T>(r, sm, a, known.row, w, W, (double)uniform * W);
    return 0;
}

template <typename T, bool RESIDENT>
__device__ void sample_row(const SampleArgs& a, Shared& sm, unsigned char* smem_raw, const SampleRest& known) {
    const int row = known.row;
    constexpr int VEC = Raw<T>::VEC, STRIDE = 32 * VEC;
    cg::cluster_group cluster = cg::this_cluster();
    const int CL = cluster.num_blocks(), me = cluster.block_rank();
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
    // next to infinite logits no other has weight: they count as 0 and the others as -infinity
    const bool infinite = isinf(known.M);
    auto only_infinite = [&](float (&x)[VEC]) {
        if (infinite)
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = x[e] == INFINITY ? 0.f : -INFINITY;
    };
    auto load = [&](int i, float (&x)[VEC]) {
        if (RESIDENT) Raw<T>::unpack(kept_row[i / VEC], x);
        else {
            fetch(i, x);
            only_infinite(x);
        }
    };

    Row r;
    const Limits l = limits_of(a, row);
    const float uniform = l.uniform, top_p = l.top_p;
    const int top_k = l.top_k;
    const bool use_k = l.use_k, use_p = l.use_p, use_m = l.use_m;

    if (tid == 0) { sm.answer = ~0ull; sm.n_list = 0; }
    if (tid < TAB) sm.tab[tid] = POW_TABLE.v[tid];
    sm.hist[tid] = 0;
    set_row(r, l, known.M);
    int bin = 0;
    __syncthreads();
    // a long front of top-p (not of a row that the list holds as it is, nor with logits so large that their last bit is 3e-5 of a weight or that a bin's number does not fit)
    if (use_p && !use_k && !use_m && a.vocab > LIST && fabsf(known.M) * r.steps < 17000.f && fabsf(known.M) < 1e7f && front_bins<T>(r, sm, a, known, top_p, bin, me, CL))
        for (int tries = 0; tries < 3; ++tries) {
            front_slices<T>(r, sm, a, known, bin, me, CL);
            cluster.sync();
            int verdict = 0;
            if (me == 0) verdict = from_front<T>(r, sm, a, known, top_p, uniform);
            if (me == 0 && tid < CL) *cluster.map_shared_rank(&sm.verdict, tid) = verdict;
            cluster.sync();
            verdict = sm.verdict;
            if (verdict == 0) return;
            if (verdict == 2) break;
            bin -= verdict;
            if (tid == 0) { sm.answer = ~0ull; sm.n_list = 0; }
            cluster.sync();
        }
    __syncthreads();
    if (tid == 0) { sm.answer = ~0ull; sm.n_list = 0; }
    sm.hist[tid] = 0;
    cluster.barrier_arrive();             // (before anybody looks into another block's shared memory, all have to have started)

    // ---- the row into shared memory, each thread's largest
    float own_best = -INFINITY;
    auto take = [&](int i, float (&x)[VEC]) {
        only_infinite(x);
        if (RESIDENT) kept_row[i / VEC] = Raw<T>::pack(x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) own_best = fmaxf(own_best, x[e]);
    };
    constexpr int AHEAD = 8;              // loads of a lane under way
    int i_load = w0 + lane * VEC;
    if (aligned)
        for (; i_load + (AHEAD - 1) * STRIDE + VEC <= w1; i_load += AHEAD * STRIDE) {
            uint4 u[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) u[j] = __ldg(reinterpret_cast<const uint4*>(logits + first + i_load + j * STRIDE));
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                float x[VEC];
                Raw<T>::unpack(u[j], x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[e] = number(x[e]);
                take(i_load + j * STRIDE, x);
            }
        }
    for (; i_load < w1; i_load += STRIDE) {
        float x[VEC];
        fetch(i_load, x);
        take(i_load, x);
    }
    cluster.barrier_wait();
    r.M = infinite ? 0.f : known.M;
    set_row(r, l, r.M);

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
#pragma unroll
            for (int w = 0; w < NW; ++w) t += sm.warp_sum[w];
            cluster.map_shared_rank(sm.sum[flip], tid)[me] = t;
        }
    };
    auto total = [&]() {
        double t = 0.0;
#pragma unroll
        for (int c = 0; c < MAX_CL; ++c) t += c < CL ? sm.sum[flip][c] : 0.0;
        return t;
    };

    // what the list's parts of the blocks come to, and where each begins; LIST + 1: too many
    int count = 0, from[MAX_CL];
    auto count_parts = [&]() {                // after a barrier of the block; has one of the cluster
        if (tid < CL) cluster.map_shared_rank(sm.n_of, tid)[me] = sm.n_list;
        cluster.sync();
        count = 0;
#pragma unroll
        for (int c = 0; c < MAX_CL; ++c) {
            from[c] = count;
            count = min(count + (int)(c < CL ? sm.n_of[c] : 0u), LIST + 1);
        }
    };
    auto fetch_parts = [&]() {                // the first block takes the others' parts behind its own
        for (int i = (int)sm.n_list + tid; i < count; i += NT) {
            int c = 1, start = from[1];
#pragma unroll
            for (int k = 2; k < MAX_CL; ++k)
                if (k < CL && i >= from[k]) { c = k; start = from[k]; }
            sm.list[i] = cluster.map_shared_rank(sm.list, c)[i - start];
        }
    };

    double S = known.S;
    if (infinite) {                       // (a weight of 1 each)
        double s = 0.0;
        for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
            float x[VEC];
            load(i, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s += x[e] == 0.f ? 1.0 : 0.0;
        }
        publish(s);
        cluster.sync();
        S = total();
    }
    if (use_k || use_p || use_m) {
        const bool weigh = use_p && !use_k;
        int last_bin = -1;                // wide bins up to here go to the list; -1: too many
        if (a.vocab <= LIST) last_bin = BINS - 1;
        else if (use_k) {
            // the threads' largest logits (equal shares of the row for each, or one element more); all of them where these are too few (us, 5 bf16 rows of 2974, top-k 1000: 66, with all 30)
            if (4 * top_k <= CL * NT) {
                const int b = wide_bin(r, own_best);
                if (b < BINS - 1) atomicAdd(&sm.hist[b], 1u);
            } else if (top_k <= LIST)
                for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                    float x[VEC];
                    load(i, x);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const int b = wide_bin(r, x[e]);
                        if (b < BINS - 1 && i + e < n) atomicAdd(&sm.hist[b], 1u);
                    }
                }
            cluster.sync();
            unsigned part[MAX_CL], mine = 0;
#pragma unroll
            for (int c = 0; c < MAX_CL; ++c) part[c] = c < CL ? cluster.map_shared_rank(sm.hist, c)[tid] : 0u;
#pragma unroll
            for (int c = 0; c < MAX_CL; ++c) mine += part[c];
            const unsigned in = warp_scan_u32(mine, lane);
            if (lane == 31) sm.warp_count[warp] = in;
            if (tid == 0) sm.bin = BINS;
            __syncthreads();
            unsigned before = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) before += w < warp ? sm.warp_count[w] : 0u;
            if (before + in >= (unsigned)top_k && before + in <= LIST) atomicMin(&sm.bin, tid);
            __syncthreads();
            if (sm.bin < BINS - 1) last_bin = sm.bin;
        } else if (!weigh) {
            const double d = -log((double)r.min_p) * 1.4426950408889634 * STEPS * 1.00001 + 1.0;
            if (d < FINE) last_bin = (int)d;
        }
        if (last_bin >= 0) {
            // each block's own part of it first
            const float cut = a.vocab <= LIST ? -INFINITY : r.M - wide_end(last_bin) / r.steps * 1.00001f;
#pragma unroll 4
            for (int i = w0 + lane * VEC; i < w1; i += STRIDE) {
                float x[VEC];
                load(i, x);
                float top = x[0];
#pragma unroll
                for (int e = 1; e < VEC; ++e) top = fmaxf(top, x[e]);
                if (!(top < cut)) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (wide_bin(r, x[e]) <= last_bin && i + e < n) {
                            const unsigned p = atomicAdd(&sm.n_list, 1u);
                            if (p < LIST) sm.list[p] = rank_of(x[e], first + i + e);
                        }
                }
            }
            __syncthreads();
            count_parts();
            if (count <= LIST) {
                if (me != 0) {
                    cluster.sync();                                // (the first block has fetched the parts)
                    return;
                }
                fetch_parts();
                cluster.barrier_arrive();
                from_list<T>(r, sm, a, row, count, use_k ? top_k : count, use_p ? top_p : 2.f, use_k ? -1.0 : S, uniform, true);
                cluster.barrier_wait();
                return;
            }
        }
        cluster.sync();                                            // histograms and counts have been read
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
            if (use_k) {
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

template <typename T, bool RESIDENT>
__global__ void __launch_bounds__(NT, 2) k_sample_rest(const __grid_constant__ SampleArgs a) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ Shared sm;
    pdl_wait();
    const int CL = cg::this_cluster().num_blocks(), count = __ldcg(a.n_rest);
    for (int i = blockIdx.x / CL; i < count; i += gridDim.x / CL) {
        sample_row<T, RESIDENT>(a, sm, smem_raw, a.rest[i]);
        __syncthreads();                  // (a warp may still have been reading the row)
    }
}

// ---- first pass: a block has a slice of a row in its registers, reads it once and leaves what the second pass needs
constexpr int SCAN_BLOCKS = 5;            // (us, 272 rows of 128256 with a nucleus each: 3 205, 4 203, 5 200)
template <typename T>
__global__ void __launch_bounds__(SCAN_THREADS, SCAN_BLOCKS) k_sample_scan(const __grid_constant__ SampleArgs a) {
    constexpr int VEC = Raw<T>::VEC, PER = SLICE / SCAN_THREADS / VEC;
    __shared__ double s_tab[TAB], s_sum[SCAN_WARPS];
    __shared__ uint32_t s_hist[BINS], s_key[SCAN_WARPS], s_index;
    __shared__ unsigned s_count[SCAN_WARPS];
    __shared__ int s_bin;
    __shared__ unsigned s_before, s_near_n;
    __shared__ float s_near[SCAN_THREADS], s_cut;
    const int row = blockIdx.x / a.slices, slice = blockIdx.x - row * a.slices, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    const T* logits = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride;
    const int first = slice * SLICE, n = min(SLICE, a.vocab - first), i0 = warp * STRETCH + lane * VEC;       // a warp has a stretch, lanes side by side
    uint4 raw[PER];
    load_slice<T>(logits + first, n, i0, raw);
    const Limits l = limits_of(a, row);
    if (tid < TAB) s_tab[tid] = POW_TABLE.v[tid];
    for (int i = tid; i < BINS; i += SCAN_THREADS) s_hist[i] = 0;
    if (tid == 0) {
        s_index = ~0u;
        s_near_n = 0;
        if (blockIdx.x == 0) *a.n_rest = 0;
    }
    auto unpack = [&](int j, float (&x)[VEC]) { Raw<T>::unpack(raw[j], x); };
    // ---- the largest
    float mine = -INFINITY;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        float x[VEC];
        unpack(j, x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            x[e] = number(x[e]);
            mine = fmaxf(mine, x[e]);
        }
        raw[j] = Raw<T>::pack(x);
    }
    const uint32_t key = __reduce_max_sync(0xffffffffu, order_key(mine));
    if (lane == 0) s_key[warp] = key;
    __syncthreads();
    uint32_t top = 0;
#pragma unroll
    for (int w = 0; w < SCAN_WARPS; ++w) top = max(top, s_key[w]);
    const float M = key_value(top);
    if (order_key(mine) == top) {
        int at = SLICE;
#pragma unroll
        for (int j = PER - 1; j >= 0; --j) {
            float x[VEC];
            unpack(j, x);
#pragma unroll
            for (int e = VEC - 1; e >= 0; --e)
                if (x[e] == M) at = i0 + j * 32 * VEC + e;
        }
        atomicMin(&s_index, (uint32_t)(first + at));
    }
    SampleSlice* out = a.slice + (size_t)row * a.slices + slice;
    Row r;
    set_row(r, l, M);
    const bool skip = l.bad || l.one || isinf(M);         // (rows with an infinite logit are the rest's)
    // ---- its weights, as far as sums over the row are asked for
    const bool weigh = !skip && !l.use_k && (l.use_p || !l.use_m);
    if (weigh) {
        double s = 0.0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            float x[VEC];
            unpack(j, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s += weight(r, s_tab, x[e]);
        }
        s = warp_sum_f64(s);
        if (lane == 0) s_sum[warp] = s;
    }
    unsigned listed = 0;
    // ---- its largest elements: the ones not below a value that so many of the threads' largest reach that `want` elements do, more or less
    float cut = INFINITY;
    if (!skip && (l.use_k || l.use_p || l.use_m)) {
        if (n <= CAP) cut = -INFINITY;
        else {
            const float share = (float)l.top_k * ((float)n / (float)a.vocab), most = fminf((float)WANT, (float)LIST / (float)a.slices);
            const float want = l.use_k ? share + 6.f * sqrtf(share) + 8.f : most;           // of the first top_k hardly ever more lie in one slice
            if (want <= (l.use_k ? 125.f : most)) {
                const int threads = n / STRETCH * 32 + min(32, (n % STRETCH + VEC - 1) / VEC);
                const unsigned of = (unsigned)fmaxf(1.f, (float)threads * (1.f - __expf(-want / (float)threads)));
                const int b = wide_bin(r, mine);
                if (b < BINS - 1) atomicAdd(&s_hist[b], 1u);
                if (tid == 0) s_bin = BINS - 1;
                __syncthreads();
                const unsigned n0 = s_hist[2 * tid], n1 = s_hist[2 * tid + 1], in = warp_scan_u32(n0 + n1, lane);
                if (lane == 31) s_count[warp] = in;
                __syncthreads();
                unsigned before = in - n0 - n1;
#pragma unroll
                for (int w = 0; w < SCAN_WARPS; ++w) before += w < warp ? s_count[w] : 0u;
                if (before < of && of <= before + n0) { s_bin = 2 * tid; s_before = before; }
                else if (before + n0 < of && of <= before + n0 + n1) { s_bin = 2 * tid + 1; s_before = before + n0; }
                __syncthreads();
                if (s_bin < BINS - 1) {
                    // of the largest in that bin the one itself
                    if (b == s_bin) s_near[atomicAdd(&s_near_n, 1u)] = mine;
                    __syncthreads();
                    if (b == s_bin) {
                        unsigned over = s_before, same = 0;
                        for (unsigned i = 0; i < s_near_n; ++i) {
                            over += s_near[i] > mine;
                            same += s_near[i] == mine;
                        }
                        if (over < of && of <= over + same) s_cut = mine;
                    }
                    __syncthreads();
                    cut = s_cut;
                    if (l.use_m && !(l.use_k && l.use_p)) {
                        // what min_p takes away from the largest here it takes away from the row's
                        const double d = -log(r.min_p) * (1.4426950408889634 * STEPS) * 1.00001 + 1.0;
                        cut = fmaxf(cut, M - (float)fmin(d, 3e38) / r.steps);
                    }
                }
            }
        }
        unsigned long long* list = a.entries + ((size_t)row * a.slices + slice) * CAP;
        if (cut < INFINITY) {
            // which of a thread's elements as bits, places in the order of the warps and lanes
            uint32_t bits = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                float x[VEC];
                unpack(j, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) bits |= (uint32_t)(x[e] >= cut && i0 + j * 32 * VEC + e < n) << (j * VEC + e);
            }
            listed = put_bits<T>(raw, bits, s_count, list, first + i0);
        }
    }
    __syncthreads();
    if (tid == 0) {
        out->best = ((unsigned long long)~top << 32) | s_index;
        out->n = listed <= CAP ? (int)listed : 0;
        out->cut = listed <= CAP ? cut : INFINITY;
    }
    if (tid < SCAN_WARPS) out->stretch[tid] = weigh ? s_sum[tid] : 0.0;
}

// ---- second pass: a block for each row; what cannot be settled from the slices' lists goes to the rest
template <typename T>
__global__ void __launch_bounds__(NT) k_sample_list(const __grid_constant__ SampleArgs a) {
    __shared__ Shared sm;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    if (tid < TAB) sm.tab[tid] = POW_TABLE.v[tid];
    sm.hist[tid] = 0;
    if (tid == 0) { sm.answer = ~0ull; sm.n_list = 0; sm.lo[0] = 0; }
    const Limits l = limits_of(a, row);
    __syncthreads();
    pdl_wait();
    const SampleSlice* slice = a.slice + (size_t)row * a.slices;
    // (slices <= NT: a thread for each)
    unsigned long long best = ~0ull;
    float cut = -INFINITY;
    int n = 0;
    if (tid < a.slices) {
        best = __ldcg(&slice[tid].best);
        cut = __ldcg(&slice[tid].cut);
        n = __ldcg(&slice[tid].n);
        sm.all[tid] = n;
    }
    unsigned long long first = best;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) first = min(first, __shfl_xor_sync(0xffffffffu, first, o));
    const uint32_t highest = __reduce_max_sync(0xffffffffu, tid < a.slices && best != ~0ull && rank_value(best) != -INFINITY ? order_key(cut) : 0u);
    if (lane == 0) {
        if (first != ~0ull) atomicMin(&sm.answer, first);
        atomicMax(&sm.lo[0], highest);
    }
    __syncthreads();
    const float M = rank_value(sm.answer);
    if (l.bad || M == -INFINITY || l.one) {
        if (tid == 0) {
            const bool none = l.bad || M == -INFINITY;
            a.tokens[row] = none ? -1 : (int)(uint32_t)sm.answer;
            if (a.logprob) a.logprob[row] = none ? __int_as_float(0x7fffffff) : 0.f;
        }
        return;
    }
    if (isinf(M)) {
        if (tid == 0) a.rest[atomicAdd(a.n_rest, 1)] = {0.0, M, row};
        return;
    }
    Row r;
    set_row(r, l, M);
    cut = key_value(sm.lo[0]);            // all elements of the row that are not below it are in the lists
    // ---- sums of the slices' weights, four stretches a thread, in terms of the row's largest
    const bool plain = !l.use_k && !l.use_p && !l.use_m, weigh = l.use_p && !l.use_k;
    double S = 0.0;
    if (plain || weigh) {
        double w[PER_STRETCH], run = 0.0;
#pragma unroll
        for (int e = 0; e < PER_STRETCH; ++e) {
            const int i = tid * PER_STRETCH + e, sl = i / SCAN_WARPS;
            w[e] = 0.0;
            // (no sums without a finite logit: 0)
            if (sl < a.slices) w[e] = __ldcg(&slice[sl].stretch[i % SCAN_WARPS]) * weight(r, sm.tab, rank_value(__ldcg(&slice[sl].best)));
            if (w[e] < 0x1p-110) w[e] = 0.0;                       // (2^10 elements that count as nothing one by one)
            run += w[e];
        }
        const double in = warp_scan_f64(run, lane);
        if (lane == 31) sm.warp_sum2[warp] = in;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NW; ++k) S += sm.warp_sum2[k];
        if (plain) {
            draw_from<T>(r, sm, a, row, w, S, (double)l.uniform * S);
            return;
        }
    }
    // ---- where the front ends; what lies in front of that, if the lists hold it
    const unsigned long long* entries = a.entries + (size_t)row * a.slices * CAP;
    const int slots = a.slices * CAP;
    auto entry = [&](int i) {                                      // ~0: none
        const int sl = i / CAP;
        return i - sl * CAP < (int)sm.all[sl] ? __ldcg(entries + i) : ~0ull;
    };
    bool done = cut == -INFINITY;                                  // everything is in the lists
    if (cut < INFINITY && l.use_m && !(l.use_k && l.use_p)) done = done || weight(r, sm.tab, cut) < r.min_p * 0.999;
    const bool whole = done;
    int last_bin = BINS - 1;
    if (cut < INFINITY && (l.use_k || l.use_p)) {
        for (int i = tid; i < slots; i += NT) {
            const unsigned long long v = entry(i);
            if (v == ~0ull || rank_value(v) < cut) continue;
            const float x = rank_value(v);
            if (weigh) {
                const float d = depth_of(r, x);
                const int b = (int)d;
                if (b < BINS - 1) atomicAdd(&sm.hist[b], __float2uint_rn(UNIT * exp2f(((float)b - d) * (1.f / STEPS))));
            } else {
                const int b = wide_bin(r, x);
                if (b < BINS - 1) atomicAdd(&sm.hist[b], 1u);
            }
        }
        __syncthreads();
        // sums along the bins: elements, or weights by what each bin's upper end weighs
        const unsigned mine = sm.hist[tid];
        const float v = weigh ? (float)mine * (1.f / UNIT) * exp2f((float)tid * (-1.f / STEPS)) : (float)mine;
        float in = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const float y = __shfl_up_sync(0xffffffffu, in, o);
            if (lane >= o) in += y;
        }
        if (lane == 31) sm.warp_f[warp] = in;
        if (tid == 0) sm.bin = BINS;
        __syncthreads();
        float before = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) before += w < warp ? sm.warp_f[w] : 0.f;
        // the border is in front of here (a little further for weights, of which these are not exact; the sorted list's sums are, and say so if it was not far enough)
        const float goal = weigh ? (float)((double)l.top_p * S) * 1.0002f : (float)l.top_k;
        if (before + in >= goal) atomicMin(&sm.bin, tid);
        __syncthreads();
        if (sm.bin < BINS - 1) {
            done = true;
            last_bin = weigh && sm.bin >= FINE ? min(FINE + (sm.bin - FINE) / COARSE, BINS - 1) : sm.bin;
        }
    }
    int count = LIST + 1;
    if (done) {
        for (int i = tid; i < slots; i += NT) {
            const unsigned long long v = entry(i);
            if (v == ~0ull || rank_value(v) < cut) continue;
            if (wide_bin(r, rank_value(v)) > last_bin) continue;
            const unsigned at = atomicAdd(&sm.n_list, 1u);
            if (at < LIST) sm.list[at] = v;
        }
        __syncthreads();
        count = (int)sm.n_list;
    }
    if (count > LIST || !from_list<T>(r, sm, a, row, count, l.use_k ? l.top_k : count, l.use_p ? l.top_p : 2.f, l.use_k ? -1.0 : S, l.uniform, whole))
        if (tid == 0) a.rest[atomicAdd(a.n_rest, 1)] = {S, M, row};
}

template <typename T>
int run(SampleArgs a, int n_sm, cudaStream_t s) {
    k_sample_scan<T><<<(unsigned)((long long)a.n_rows * a.slices), SCAN_THREADS, 0, s>>>(a);
    if (launch_k(k_sample_list<T>, dim3(a.n_rows), dim3(NT), 0, s, true, a) != cudaSuccess) return -1;
    constexpr int STRIDE = 32 * Raw<T>::VEC;
    // Clusters of eight are soonest done with one row (16 slices at a time: 43 us for a call of one row of 128256; in two rounds 55), of four with many, as one block of a cluster orders the list
    // while the others wait: where a fifth of the rows may be more than there are clusters of eight (272 rows of which 55 come here: 187 us with eight, 157 with four).
    const int most = a.n_rows > 5 * (2 * n_sm / MAX_CL) ? MAX_CL / 2 : MAX_CL;
    int cl = 1;
    while (cl < most && a.vocab > cl * 4096) cl *= 2;
    a.chunk = ((a.vocab + cl - 1) / cl + STRIDE - 1) / STRIDE * STRIDE;
    // (a nearly flat row has all the elements of a block's slices in one bin)
    a.unit = (float)sample_unit((unsigned)((a.slices + 2 * cl - 1) / (2 * cl) * 2 * SLICE));
    a.per_unit = 1.f / a.unit;
    const size_t bytes = (size_t)a.chunk * sizeof(T);
    const bool resident = bytes <= SMEM_ROW;
    const int clusters = 2 * n_sm / cl < a.n_rows ? 2 * n_sm / cl : a.n_rows;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)clusters * cl);
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = resident ? bytes : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cl;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    if (resident) {
        if (ensure_dynamic_smem(reinterpret_cast<const void*>(&k_sample_rest<T, true>), SMEM_ROW)) return -1;
        return cudaLaunchKernelEx(&cfg, k_sample_rest<T, true>, a) != cudaSuccess;
    }
    return cudaLaunchKernelEx(&cfg, k_sample_rest<T, false>, a) != cudaSuccess;
}

}  // namespace

int launch_sample(int dtype, SampleArgs a, int n_sm, cudaStream_t s) {
    return dtype == 0 ? run<float>(a, n_sm, s) : run<__nv_bfloat16>(a, n_sm, s);
}

}  // namespace esp

using namespace esp;

extern "C" {

// scratch layout: [rows][slices] SampleSlice, [rows][slices][SAMPLE_CAP] entries, [rows] the rest, how many
int esp_sample_scratch_bytes(int32_t n_rows, int32_t vocab, size_t* bytes_out) {
    if (!bytes_out || n_rows < 0 || n_rows > (1 << 24) || vocab < 1 || vocab > MAX_VOCAB) return ESP_E_ARG;
    const size_t slices = (size_t)n_rows * ((vocab + SAMPLE_SLICE - 1) / SAMPLE_SLICE);
    *bytes_out = slices * (sizeof(SampleSlice) + SAMPLE_CAP * sizeof(unsigned long long)) + (size_t)n_rows * sizeof(SampleRest) + sizeof(int32_t);
    return ESP_OK;
}

int esp_sample(int32_t dtype, int32_t n_rows, int32_t vocab, const void* logits, int64_t row_stride, const esp_sampling* sampling, const float* uniform,
               int32_t* tokens, float* logprob, void* scratch, size_t scratch_bytes, void* cuda_stream) {
    if (dtype != 0 && dtype != 1) return ESP_E_BADCFG;
    const int size = dtype == 0 ? 4 : 2;
    auto off = [](const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; };
    if (n_rows < 0 || n_rows > (1 << 24) || vocab < 1 || vocab > MAX_VOCAB || row_stride < 0 || row_stride > ((int64_t)1 << 40) || !sampling) return ESP_E_ARG;
    if (off(logits, size) || off(sampling->temperature, 4) || off(sampling->top_k, 4) || off(sampling->top_p, 4) || off(sampling->min_p, 4) || off(uniform, 4) ||
        off(tokens, 4) || off(logprob, 4)) return ESP_E_ARG;
    if (n_rows == 0) return ESP_OK;
    if ((int64_t)n_rows * ((vocab + SAMPLE_SLICE - 1) / SAMPLE_SLICE) > 0x7fffffff) return ESP_E_ARG;
    if (!logits || !uniform || !tokens) return ESP_E_ARG;
    size_t need = 0;
    if (const int rc = esp_sample_scratch_bytes(n_rows, vocab, &need)) return rc;
    if (!scratch || scratch_bytes < need || off(scratch, 256)) return ESP_E_WORKSPACE;
    const int n_sm = current_sm_count();
    if (n_sm < 1) return ESP_E_CUDA;
    SampleArgs a;
    a.slices = (vocab + SAMPLE_SLICE - 1) / SAMPLE_SLICE;
    a.slice = reinterpret_cast<SampleSlice*>(scratch);
    a.entries = reinterpret_cast<unsigned long long*>(a.slice + (size_t)n_rows * a.slices);
    a.rest = reinterpret_cast<SampleRest*>(a.entries + (size_t)n_rows * a.slices * SAMPLE_CAP);
    a.n_rest = reinterpret_cast<int32_t*>(a.rest + n_rows);
    a.logits = logits; a.row_stride = row_stride; a.n_rows = n_rows; a.vocab = vocab;
    a.temperature = sampling->temperature; a.top_k = sampling->top_k; a.top_p = sampling->top_p; a.min_p = sampling->min_p;
    a.uniform = uniform; a.tokens = tokens; a.logprob = logprob; a.chunk = 0; a.unit = a.per_unit = 0.f;
    const int rc = launch_sample(dtype, a, n_sm, reinterpret_cast<cudaStream_t>(cuda_stream));
    const cudaError_t e = cudaGetLastError();
    return rc ? ESP_E_CUDA : (e == cudaSuccess ? ESP_OK : ESP_E_CUDA);
}

}  // extern "C"
