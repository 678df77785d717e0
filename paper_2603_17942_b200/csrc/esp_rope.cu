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
    for (int b0 = 0; b0 < q.batch; b0 += 32) {
        bool mine = false;
        paged::Seq s;
        if (b0 + lane < q.batch) {
            s = paged::load_seq(q, b0 + lane);
            mine = t >= s.start && t < s.start + s.n;
        }
        const uint32_t who = __ballot_sync(0xffffffffu, mine);
        if (!who) continue;
        const int src = __ffs(who) - 1;
        if (lane == src) {
            r.pos = s.kv - s.n + (t - s.start);
            if (r.pos >= 0) {
                const int index = r.pos / pages.page_size;
                r.page = paged::load_page(q, pages, b0 + lane, index);
                r.slot = r.pos - index * pages.page_size;
            }
        }
        r.page = __shfl_sync(0xffffffffu, r.page, src);
        r.slot = __shfl_sync(0xffffffffu, r.slot, src);
        r.pos = __shfl_sync(0xffffffffu, r.pos, src);
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

}  // namespace

void launch_rope_table(const uint64_t* freq, int pairs, uint64_t* table, cudaStream_t s) {
    RopeFreqs r;
    for (int i = 0; i < ESP_ROPE_MAX_DIM / 2; ++i) r.f[i] = i < pairs ? freq[i] : 0;
    k_rope_table_paged<<<1, ESP_ROPE_MAX_DIM / 2, 0, s>>>(r, pairs, table);
}

int launch_norm_rope(int dtype, const NormRopeArgs& a, cudaStream_t s) {
    const long long tasks = (long long)a.n_tokens * (a.q.n + a.k.n + a.v.n);
    const long long blocks = (tasks + ANY_WARPS - 1) / ANY_WARPS;
    if (blocks > 0x7fffffff) return -1;
    if (dtype == 0) k_norm_rope_any<float><<<(unsigned)blocks, ANY_WARPS * 32, 0, s>>>(a);
    else k_norm_rope_any<__nv_bfloat16><<<(unsigned)blocks, ANY_WARPS * 32, 0, s>>>(a);
    return 0;
}

}  // namespace esp
