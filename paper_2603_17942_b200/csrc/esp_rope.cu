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

// Heads of 32, 64, 128 or 256 elements on 16 bytes (rotated halves of whole groups of four): a lane has four pairs of a head, LH lanes a
// head, a block a few tokens or some heads of one; a thread has the same pairs of up to ROUNDS heads of its token.  In halves the
// lane's elements are four neighbours of each half, so that both members of a pair are its own; what is not rotated is halved likewise.
// Memory bounds it, next to it the instructions (a lane that had eight neighbours and its partners' values by shuffle needed 333 per eight
// elements and 65 us for 8192 tokens of 40 heads of 128), so the loads of all of a thread's heads are requested first; while they are on
// their way the tokens' slots are looked up, a warp for each, and their angles turned, once for all heads.
constexpr int ROPE_THREADS = 384;       // threads of a block at most
constexpr int ROPE_PAIRS = 1024;        // angles a block keeps
constexpr int ROPE_TOKENS = 16;         // tokens of a block at most
template <typename T> constexpr int ROPE_ROUNDS = sizeof(T) == 2 ? 4 : 2;      // heads of a thread: 64 bytes under way

template <typename T> struct Vec4;
template <> struct Vec4<__nv_bfloat16> {
    uint2 x;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { x = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint2*>(p) = x; }
    __device__ __forceinline__ void get(float (&v)[4]) const {
        v[0] = __uint_as_float(x.x << 16); v[1] = __uint_as_float(x.x & 0xffff0000u);
        v[2] = __uint_as_float(x.y << 16); v[3] = __uint_as_float(x.y & 0xffff0000u);
    }
    __device__ __forceinline__ void set(const float (&v)[4]) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
        x = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
};
template <> struct Vec4<float> {
    float4 x;
    __device__ __forceinline__ void load(const float* p) { x = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = x; }
    __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; }
    __device__ __forceinline__ void set(const float (&v)[4]) { x = make_float4(v[0], v[1], v[2], v[3]); }
};

template <typename T, int LH, bool APPEND, bool INTER>
__global__ void __launch_bounds__(ROPE_THREADS, 3) k_norm_rope(const __grid_constant__ NormRopeArgs a, int heads_per_block, int heads_per_round, int tokens_per_block) {
    constexpr int ROUNDS = ROPE_ROUNDS<T>, D = LH * 8;
    __shared__ __align__(16) float2 s_turn[ROPE_PAIRS];       // [token of the block][pair]
    __shared__ Slot s_slot[ROPE_TOKENS];
    const int t0 = blockIdx.x * tokens_per_block, n_tok = min(tokens_per_block, a.n_tokens - t0);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, l = tid % LH;
    const int h0 = blockIdx.y * heads_per_block, h_end = min(h0 + heads_per_block, a.q.n + a.k.n + a.v.n);
    const int tk = tid / (heads_per_round * LH), hg = h0 + (tid - tk * heads_per_round * LH) / LH, t = t0 + tk;
    const bool mine = tk < n_tok;
    // the lane's two groups of four elements, and whether they are pairs that turn
    const int j = l * 4;
    const bool turns = j < a.pairs;
    const int o1 = INTER ? 2 * j : (turns ? j : a.pairs + j), o2 = INTER ? 2 * j + 4 : (turns ? a.pairs + j : D / 2 + j);
    const int k0 = a.q.n, v0 = a.q.n + a.k.n;
    Vec4<T> x1[ROUNDS], x2[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int h = hg + r * heads_per_round;
        if (mine && h < h_end) {
            const HeadsView& in = h < k0 ? a.q : (h < v0 ? a.k : a.v);
            const T* p = reinterpret_cast<const T*>(in.p) + paged::out_offset(in, t, h - (h < k0 ? 0 : (h < v0 ? k0 : v0)));
            x1[r].load(p + o1);
            x2[r].load(p + o2);
        }
    }
    if (APPEND) {
        for (int k = warp; k < n_tok; k += blockDim.x >> 5) {
            const Slot slot = find_slot(a.seq, a.pages, t0 + k, lane);
            if (lane == 0) s_slot[k] = slot;
        }
        if (!a.positions) __syncthreads();       // the angles wait for the slots
    }
    const int kept = (a.pairs + 3) & ~3;
    for (int i = tid; i < n_tok * a.pairs; i += blockDim.x) {
        const int k = i / a.pairs, pair = i - k * a.pairs;
        s_turn[k * kept + pair] = rope_turn(a.positions ? __ldg(a.positions + t0 + k) : s_slot[k].pos, __ldg(a.freq + pair), a.amplitude);
    }
    __syncthreads();
    float c[4], s[4];
    Slot slot;
    slot.page = slot.slot = 0;
    bool valid = mine;
    if (mine) {
        if (APPEND) {
            slot = s_slot[tk];
            valid = slot.page >= 0;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 cs = j + e < a.pairs ? s_turn[tk * kept + j + e] : make_float2(1.f, 0.f);
            c[e] = cs.x;
            s[e] = cs.y;
        }
    }
    if (__all_sync(0xffffffffu, !valid)) return;
    Vec4<T> gq1, gq2, gk1, gk2;
    const T *gq = reinterpret_cast<const T*>(a.q_gain), *gk = reinterpret_cast<const T*>(a.k_gain);
    if (gq) { gq1.load(gq + o1); gq2.load(gq + o2); }
    if (gk) { gk1.load(gk + o1); gk2.load(gk + o2); }
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int h = hg + r * heads_per_round;
        const bool here = valid && h < h_end;
        if (__all_sync(0xffffffffu, !here)) break;
        const bool is_q = h < k0, is_v = h >= v0;
        float u[4], w[4];
        x1[r].get(u);
        x2[r].get(w);
        if (gq || gk) {
            float sq = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) sq = fmaf(w[e], w[e], fmaf(u[e], u[e], sq));
#pragma unroll
            for (int o = LH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
            if (is_q ? gq != nullptr : (!is_v && gk)) {
                const float root = rsqrtf(sq * (1.f / D) + a.eps);
                float f[4];
                (is_q ? gq1 : gk1).get(f);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = u[e] * root * f[e];
                (is_q ? gq2 : gk2).get(f);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = w[e] * root * f[e];
            }
        }
        if (!here) continue;
        T* y;
        if (APPEND && !is_q) {
            const int head = h - (is_v ? v0 : k0);
            y = reinterpret_cast<T*>(is_v ? a.pages.v : a.pages.k) + (slot.page * a.pages.page + slot.slot * a.pages.tok + head * a.pages.head);
        } else {
            const HeadsView& to = is_q ? a.q_out : a.k_out;
            y = reinterpret_cast<T*>(to.p) + paged::out_offset(to, t, h - (is_q ? 0 : k0));
        }
        if (!is_v) {                             // values go as they are
            if (INTER) {
                // pairs (u0, u1), (u2, u3), (w0, w1), (w2, w3)
                float p[8] = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = p[2 * e], z = p[2 * e + 1];
                    p[2 * e] = j + e < a.pairs ? fmaf(x, c[e], -(z * s[e])) : x;
                    p[2 * e + 1] = j + e < a.pairs ? fmaf(z, c[e], x * s[e]) : z;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) { u[e] = p[e]; w[e] = p[4 + e]; }
            } else if (turns) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = u[e], z = w[e];
                    u[e] = fmaf(x, c[e], -(z * s[e]));
                    w[e] = fmaf(z, c[e], x * s[e]);
                }
            }
            x1[r].set(u);
            x2[r].set(w);
        }
        x1[r].store(y + o1);
        x2[r].store(y + o2);
    }
}

template <typename T, int LH>
void run_norm_rope(const NormRopeArgs& a, cudaStream_t s) {
    constexpr int ROUNDS = ROPE_ROUNDS<T>;
    const int heads = a.q.n + a.k.n + a.v.n, small = 128 / LH;
    int hb, per, tokens = 1;             // heads of a block and of a round, tokens of a block
    if ((long long)a.n_tokens * ((heads + small - 1) / small) <= 4 * 148) {
        // a call that does not fill the GPU spreads its heads over the SMs, a head per thread group
        hb = per = heads < small ? heads : small;
    } else {
        const int most = ROUNDS * (ROPE_THREADS / LH), parts = (heads + most - 1) / most;
        hb = (heads + parts - 1) / parts;
        per = (hb + ROUNDS - 1) / ROUNDS;
        // as many tokens as a block has threads for, but a block for every SM twice over
        tokens = ROPE_THREADS / (per * LH);
        if (tokens > ROPE_TOKENS) tokens = ROPE_TOKENS;
        const int kept = (a.pairs + 3) & ~3;
        if (kept && tokens > ROPE_PAIRS / kept) tokens = ROPE_PAIRS / kept;
        if (tokens > a.n_tokens / (2 * 148)) tokens = a.n_tokens / (2 * 148);
        if (tokens < 1) tokens = 1;
    }
    const int threads = (tokens * per * LH + 31) / 32 * 32;
    const dim3 grid((a.n_tokens + tokens - 1) / tokens, (heads + hb - 1) / hb);
    const bool inter = a.pairs && a.interleaved;
    if (a.append) {
        if (inter) k_norm_rope<T, LH, true, true><<<grid, threads, 0, s>>>(a, hb, per, tokens);
        else k_norm_rope<T, LH, true, false><<<grid, threads, 0, s>>>(a, hb, per, tokens);
    } else {
        if (inter) k_norm_rope<T, LH, false, true><<<grid, threads, 0, s>>>(a, hb, per, tokens);
        else k_norm_rope<T, LH, false, false><<<grid, threads, 0, s>>>(a, hb, per, tokens);
    }
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
    if (a.pairs && !a.interleaved && a.pairs % 4) return false;
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
