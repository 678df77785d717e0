// Per-head RMSNorm with the rotation of positions, into a tensor or into the pages of a cache.
//
//   y = x * gain / sqrt(mean(x^2) + eps);   pair (y_a, y_b) -> A (y_a c - y_b s, y_b c + y_a s),  c + i s = e^(i p f)
//
// The angle p f is taken modulo one turn in whole numbers: the table holds f / 2 pi as a 64-bit fraction of a turn, p times it
// wraps around by itself, and the upper 32 bits are the angle to 2^-32 of a turn for every 32-bit position.  (p * f in fp32
// would be off by 0.06 rad at p = 10^6 for the fastest pair.)
#include "esp_paged.cuh"

namespace esp {

namespace {

struct RopeFreqs {
    uint64_t f[ESP_ROPE_MAX_DIM / 2];
};
__global__ void k_rope_table_paged(const __grid_constant__ RopeFreqs r, int pairs, uint64_t* table) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < pairs) table[i] = r.f[i];
}

// (A cos, A sin) of position p's angle.  (int32) of the upper word is the angle in 2^-31 half turns, in [-1, 1).
__device__ __forceinline__ float2 rope_turn(int p, uint64_t f, float amplitude) {
    const uint64_t turns = (uint64_t)(int64_t)p * f;
    float s, c;
    sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, &s, &c);
    return make_float2(amplitude * c, amplitude * s);
}

// Where token t of the call goes: its sequence's slot.  page < 0: nowhere.  Called by whole warps.
struct Slot {
    int page, slot, pos;
};
__device__ __forceinline__ Slot find_slot(const SeqTable& q, const PagesView& pages, int t, int lane) {
    Slot r;
    r.page = -1;
    r.slot = r.pos = 0;
    for (int b0 = 0; b0 < q.batch; b0 += 128) {
        int b = -1, first = 0;                         // this lane's sequence, position of its first new token minus the token's number
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = b0 + 32 * i + lane;
            if (x < q.batch) {
                const paged::Seq s = paged::load_seq(q, x);
                if (t >= s.start && t < s.start + s.n) { b = x; first = s.kv - s.n - s.start; }
            }
        }
        const uint32_t who = __ballot_sync(0xffffffffu, b >= 0);
        if (!who) continue;
        const int src = __ffs(who) - 1;
        b = __shfl_sync(0xffffffffu, b, src);
        r.pos = __shfl_sync(0xffffffffu, first, src) + t;
        if (r.pos >= 0) {
            const int index = r.pos / pages.page_size;
            r.page = paged::load_page(q, pages, b, index);
            r.slot = r.pos - index * pages.page_size;
        }
        break;
    }
    return r;
}

// Any head size, stride, alignment and rotated share: a warp takes one head of one token, its elements 32 apart in the lanes; the
// normed row stands in shared memory, where a lane finds the partner of its element.  Everything is read before anything is written,
// so that the output may be the input.
constexpr int ANY_WARPS = 8, ANY_PER_LANE = ESP_ROPE_MAX_DIM / 32;

template <typename T>
__global__ void __launch_bounds__(ANY_WARPS * 32) k_norm_rope_any(const __grid_constant__ NormRopeArgs a) {
    __shared__ float rows[ANY_WARPS][ESP_ROPE_MAX_DIM];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int heads = a.q.n + a.k.n + a.v.n;
    const long long task = (long long)blockIdx.x * ANY_WARPS + warp;
    if (task >= (long long)a.n_tokens * heads) return;
    const int t = (int)(task / heads);
    int h = (int)(task - (long long)t * heads);
    const int kind = h < a.q.n ? 0 : (h < a.q.n + a.k.n ? 1 : 2);
    const HeadsView& in = kind == 0 ? a.q : (kind == 1 ? a.k : a.v);
    const HeadsView& to = kind == 0 ? a.q_out : a.k_out;
    h -= kind == 0 ? 0 : (kind == 1 ? a.q.n : a.q.n + a.k.n);

    Slot slot;
    slot.page = slot.slot = slot.pos = 0;
    if (a.append) {
        slot = find_slot(a.seq, a.pages, t, lane);
        if (slot.page < 0) return;
    }
    const T* x = reinterpret_cast<const T*>(in.p) + paged::out_offset(in, t, h);
    T* y = kind == 0 || !a.append
               ? reinterpret_cast<T*>(to.p) + paged::out_offset(to, t, h)
               : reinterpret_cast<T*>(kind == 1 ? a.pages.k : a.pages.v) + (slot.page * a.pages.page + slot.slot * a.pages.tok + h * a.pages.head);
    const T* gain = reinterpret_cast<const T*>(kind == 0 ? a.q_gain : a.k_gain);
    T raw[ANY_PER_LANE];
    float v[ANY_PER_LANE], sq = 0.f;
#pragma unroll
    for (int i = 0; i < ANY_PER_LANE; ++i) {
        const int d = lane + 32 * i;
        raw[i] = d < a.D ? x[d] : from_f32<T>(0.f);
        v[i] = to_f32(raw[i]);
        sq = fmaf(v[i], v[i], sq);
    }
    if (kind == 2) {                  // values go as they are
#pragma unroll
        for (int i = 0; i < ANY_PER_LANE; ++i)
            if (lane + 32 * i < a.D) y[lane + 32 * i] = raw[i];
        return;
    }
    if (gain) {
        const float r = rsqrtf(warp_sum(sq) / (float)a.D + a.eps);
#pragma unroll
        for (int i = 0; i < ANY_PER_LANE; ++i)
            if (lane + 32 * i < a.D) v[i] = v[i] * r * to_f32(gain[lane + 32 * i]);
    }
#pragma unroll
    for (int i = 0; i < ANY_PER_LANE; ++i)
        if (lane + 32 * i < a.D) rows[warp][lane + 32 * i] = v[i];
    __syncwarp();
    const int p = a.positions ? __ldg(a.positions + t) : slot.pos;
#pragma unroll
    for (int i = 0; i < ANY_PER_LANE; ++i) {
        const int d = lane + 32 * i;
        if (d >= a.D) break;
        float o = v[i];
        if (d < 2 * a.pairs) {
            const int pair = a.interleaved ? d >> 1 : (d < a.pairs ? d : d - a.pairs);
            const bool second = a.interleaved ? (d & 1) : d >= a.pairs;
            const float other = rows[warp][a.interleaved ? d ^ 1 : (second ? d - a.pairs : d + a.pairs)];
            const float2 cs = rope_turn(p, __ldg(a.freq + pair), a.amplitude);
            o = second ? fmaf(o, cs.x, other * cs.y) : fmaf(o, cs.x, -(other * cs.y));
        }
        y[d] = from_f32<T>(o);
    }
}

// Heads of 32, 64, 128 or 256 elements on 16 bytes (rotated halves of whole groups of eight): a lane has eight neighbouring elements, LH lanes a
// head, a block a token or some of its heads.  Memory bounds it, so the loads of all of a thread's heads (the same elements of each)
// are requested first; while they are on their way one warp looks up the token's slot and the others turn its angles, once for all heads.
constexpr int ROPE_ROUNDS = 4;          // heads of a thread
constexpr int ROPE_THREADS = 384;       // threads of a block at most

template <typename T> struct Vec8;
template <> struct Vec8<__nv_bfloat16> {
    uint4 x;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { x = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = x; }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void set(const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]); w[i] = *reinterpret_cast<const uint32_t*>(&b); }
        x = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec8<float> {
    float4 x, y;
    __device__ __forceinline__ void load(const float* p) { x = reinterpret_cast<const float4*>(p)[0]; y = reinterpret_cast<const float4*>(p)[1]; }
    __device__ __forceinline__ void store(float* p) const { reinterpret_cast<float4*>(p)[0] = x; reinterpret_cast<float4*>(p)[1] = y; }
    __device__ __forceinline__ void get(float (&v)[8]) const { v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w; }
    __device__ __forceinline__ void set(const float (&v)[8]) { x = make_float4(v[0], v[1], v[2], v[3]); y = make_float4(v[4], v[5], v[6], v[7]); }
};

template <typename T, int LH, bool APPEND>
__global__ void __launch_bounds__(ROPE_THREADS) k_norm_rope(const __grid_constant__ NormRopeArgs a, int heads_per_block) {
    __shared__ float2 turn[LH * 4];     // the token's pairs
    __shared__ Slot s_slot;
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, l = tid % LH;
    const int h0 = blockIdx.y * heads_per_block, n_heads = min(heads_per_block, a.q.n + a.k.n + a.v.n - h0), per_round = blockDim.x / LH;
    Vec8<T> x[ROPE_ROUNDS];
#pragma unroll
    for (int r = 0; r < ROPE_ROUNDS; ++r) {
        const int i = tid / LH + r * per_round;
        if (i < n_heads) {
            int h = h0 + i;
            const HeadsView& in = h < a.q.n ? a.q : (h < a.q.n + a.k.n ? a.k : a.v);
            h -= h < a.q.n ? 0 : (h < a.q.n + a.k.n ? a.q.n : a.q.n + a.k.n);
            x[r].load(reinterpret_cast<const T*>(in.p) + paged::out_offset(in, t, h) + l * 8);
        }
    }
    Slot slot;
    slot.page = slot.slot = slot.pos = 0;
    if (APPEND) {
        if (warp == 0) {
            slot = find_slot(a.seq, a.pages, t, lane);
            if (lane == 0) s_slot = slot;
        }
        if (!a.positions) {              // the angles wait for the slot
            __syncthreads();
            slot = s_slot;
        }
    }
    if (a.pairs) {
        const int p = a.positions ? __ldg(a.positions + t) : slot.pos;
        for (int i = tid; i < a.pairs; i += blockDim.x) turn[i] = rope_turn(p, __ldg(a.freq + i), a.amplitude);
    }
    __syncthreads();
    if (APPEND) {
        slot = s_slot;
        if (slot.page < 0) return;
    }
    // the pairs of this lane's elements: in halves, eight of the first elements or eight of the second ones; else four whole pairs
    const int shift = a.pairs / 8;       // lanes between a pair's halves
    const bool first = l < shift, second = !first && l < 2 * shift;
#pragma unroll
    for (int r = 0; r < ROPE_ROUNDS; ++r) {
        const int i = tid / LH + r * per_round;
        if (__all_sync(0xffffffffu, i >= n_heads)) break;
        const bool valid = i < n_heads;
        int h = valid ? h0 + i : h0;
        const int kind = h < a.q.n ? 0 : (h < a.q.n + a.k.n ? 1 : 2);
        h -= kind == 0 ? 0 : (kind == 1 ? a.q.n : a.q.n + a.k.n);
        float v[8];
        if (!valid) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
        } else {
            x[r].get(v);
        }
        const T* gain = reinterpret_cast<const T*>(kind == 0 ? a.q_gain : (kind == 1 ? a.k_gain : nullptr));
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = fmaf(v[e], v[e], sq);
#pragma unroll
        for (int o = LH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
        if (gain) {
            const float root = rsqrtf(sq / (float)(LH * 8) + a.eps);
            Vec8<T> gv;
            gv.load(gain + l * 8);
            float gf[8];
            gv.get(gf);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = v[e] * root * gf[e];
        }
        if (a.pairs && a.interleaved) {
            if (kind < 2) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (l * 4 + e < a.pairs) {
                        const float2 cs = turn[l * 4 + e];
                        const float p = v[2 * e], q = v[2 * e + 1];
                        v[2 * e] = fmaf(p, cs.x, -(q * cs.y));
                        v[2 * e + 1] = fmaf(q, cs.x, p * cs.y);
                    }
                }
            }
        } else if (a.pairs) {
            const int src = first ? l + shift : (second ? l - shift : l);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float other = __shfl_sync(0xffffffffu, v[e], src, LH);
                if (kind < 2 && (first || second)) {
                    const float2 cs = turn[(first ? l : l - shift) * 8 + e];
                    v[e] = first ? fmaf(v[e], cs.x, -(other * cs.y)) : fmaf(v[e], cs.x, other * cs.y);
                }
            }
        }
        if (!valid) continue;
        T* y;
        if (APPEND && kind) y = reinterpret_cast<T*>(kind == 1 ? a.pages.k : a.pages.v) + (slot.page * a.pages.page + slot.slot * a.pages.tok + h * a.pages.head);
        else {
            const HeadsView& to = kind == 0 ? a.q_out : a.k_out;
            y = reinterpret_cast<T*>(to.p) + paged::out_offset(to, t, h);
        }
        if (kind < 2) x[r].set(v);       // values go as they are
        x[r].store(y + l * 8);
    }
}

template <typename T, int LH>
void run_norm_rope(const NormRopeArgs& a, cudaStream_t s) {
    const int heads = a.q.n + a.k.n + a.v.n;
    // a call that does not fill the GPU spreads its heads over the SMs, a head per thread group
    const int small = 128 / LH;
    int hb, threads;
    if ((long long)a.n_tokens * ((heads + small - 1) / small) <= 4 * 148) {
        hb = heads < small ? heads : small;
        threads = (hb * LH + 31) / 32 * 32;
    } else {
        const int parts = (heads * LH + ROPE_ROUNDS * ROPE_THREADS - 1) / (ROPE_ROUNDS * ROPE_THREADS);
        hb = (heads + parts - 1) / parts;
        const int rounds = (hb * LH + ROPE_THREADS - 1) / ROPE_THREADS;
        threads = ((hb * LH + rounds - 1) / rounds + 31) / 32 * 32;
    }
    const dim3 grid(a.n_tokens, (heads + hb - 1) / hb);
    if (a.append) k_norm_rope<T, LH, true><<<grid, threads, 0, s>>>(a, hb);
    else k_norm_rope<T, LH, false><<<grid, threads, 0, s>>>(a, hb);
}
template <typename T>
void run_norm_rope_d(const NormRopeArgs& a, cudaStream_t s) {
    if (a.D == 32) run_norm_rope<T, 4>(a, s);
    else if (a.D == 64) run_norm_rope<T, 8>(a, s);
    else if (a.D == 128) run_norm_rope<T, 16>(a, s);
    else run_norm_rope<T, 32>(a, s);
}
bool fast_shape(const NormRopeArgs& a, int elem) {
    if (a.D != 32 && a.D != 64 && a.D != 128 && a.D != 256) return false;
    if (a.pairs && !a.interleaved && a.pairs % 8) return false;
    const int per16 = 16 / elem;
    auto al = [&](const HeadsView& v) { return !v.p || (reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.tok % per16 == 0 && v.head % per16 == 0); };
    auto al_p = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    if (!al(a.q) || !al(a.k) || !al(a.v) || !al(a.q_out) || !al(a.k_out) || !al_p(a.q_gain) || !al_p(a.k_gain)) return false;
    return !a.append || (al_p(a.pages.k) && al_p(a.pages.v) && a.pages.page % per16 == 0 && a.pages.tok % per16 == 0 && a.pages.head % per16 == 0);
}

}  // namespace

void launch_rope_table(const uint64_t* freq, int pairs, uint64_t* table, cudaStream_t s) {
    RopeFreqs r;
    for (int i = 0; i < ESP_ROPE_MAX_DIM / 2; ++i) r.f[i] = i < pairs ? freq[i] : 0;
    k_rope_table_paged<<<1, ESP_ROPE_MAX_DIM / 2, 0, s>>>(r, pairs, table);
}

int launch_norm_rope(int dtype, const NormRopeArgs& a, cudaStream_t s) {
    const int heads = a.q.n + a.k.n + a.v.n;
    if (fast_shape(a, dtype == 0 ? 4 : 2) && heads <= 65535) {
        if (dtype == 0) run_norm_rope_d<float>(a, s);
        else run_norm_rope_d<__nv_bfloat16>(a, s);
        return 0;
    }
    const long long tasks = (long long)a.n_tokens * heads;
    const long long blocks = (tasks + ANY_WARPS - 1) / ANY_WARPS;
    if (blocks > 0x7fffffff) return -1;
    if (dtype == 0) k_norm_rope_any<float><<<(unsigned)blocks, ANY_WARPS * 32, 0, s>>>(a);
    else k_norm_rope_any<__nv_bfloat16><<<(unsigned)blocks, ANY_WARPS * 32, 0, s>>>(a);
    return 0;
}

}  // namespace esp
