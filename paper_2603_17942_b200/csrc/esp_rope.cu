// Per-head RMSNorm with the rotation of positions, into a tensor or into the pages of a cache.
//
//   y = x * gain / sqrt(mean(x^2) + eps);   pair (y_a, y_b) -> A (y_a c - y_b s, y_b c + y_a s),  c + i s = e^(i p f)
//
// The angle p f is taken modulo one turn in whole numbers: the table holds f / 2 pi as a 64-bit fraction of a turn, p times it
// wraps around by itself, and the upper 32 bits are the angle to 2^-31 of a turn for every 32-bit position.  (p * f in fp32
// would be off by 0.06 rad at p = 10^6 for the fastest pair.)  The sine takes it in fp32: 24 bits of at most half a turn, off by 2^-26 of a turn or 9.4e-8 rad at
// most, about the rounding that an fp32 result has anyway.
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

// (A cos, A sin) of position p's angle.  (int32) of the upper word is the angle in 2^-31 half turns, in [-1, 1); the float keeps 24 bits of it.
__device__ __forceinline__ float2 rope_turn(int p, uint64_t f, float amplitude) {
    const uint64_t turns = (uint64_t)(int64_t)p * f;
    float s, c;
    sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, &s, &c);
    return make_float2(amplitude * c, amplitude * s);
}

// Token t's sequence in a batch where some do not hold together (see load_seq) and the position of its first new token minus that token's number; x < 0: none.
__device__ __forceinline__ int2 find_among_odd(const SeqTable& q, int t, int lane) {
    int before = 0;                                    // furthest end of the sequences of earlier rounds
    for (int b0 = 0; b0 < q.batch; b0 += 32) {
        const int x = b0 + lane;
        int end = 0, first = 0;
        bool odd, here = false;
        paged::Seq s;
        s.start = 0;
        if (x < q.batch) {
            s = paged::load_seq(q, x, end, odd);
            here = t >= s.start && t < s.start + s.n;
            first = s.kv - s.n - s.start;
        }
        const int top = max(before, paged::warp_max_before(end, lane));
        const uint32_t who = __ballot_sync(0xffffffffu, here && s.start >= top);
        if (who) {
            const int src = __ffs(who) - 1;
            return make_int2(b0 + src, __shfl_sync(0xffffffffu, first, src));
        }
        before = max(before, __reduce_max_sync(0xffffffffu, end));
    }
    return make_int2(-1, 0);
}
// Where token t of the call goes: its sequence's slot.  page < 0: nowhere.  Called by whole warps.
struct Slot {
    int page, slot, pos;
};
__device__ __forceinline__ Slot find_slot(const SeqTable& q, const PagesView& pages, int t, int lane) {
    Slot r;
    r.page = -1;
    r.slot = r.pos = 0;
    bool odd = false;
    for (int b0 = 0; b0 < q.batch; b0 += 128) {
        int b = -1, first = 0;                         // this lane's sequence, position of its first new token minus the token's number
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = b0 + 32 * i + lane;
            if (x < q.batch) {
                int top = 0;
                const paged::Seq s = paged::load_seq(q, x, top, odd);
                if (t >= s.start && t < s.start + s.n) { b = x; first = s.kv - s.n - s.start; }
            }
        }
        const uint32_t who = __ballot_sync(0xffffffffu, b >= 0);
        if (!who) continue;
        const int src = __ffs(who) - 1;
        b = __shfl_sync(0xffffffffu, b, src);
        first = __shfl_sync(0xffffffffu, first, src);
        if (__any_sync(0xffffffffu, odd)) {
            const int2 found = find_among_odd(q, t, lane);
            b = found.x;
            first = found.y;
            if (b < 0) break;
        }
        r.pos = first + t;
        if (r.pos >= 0) {
            const int index = paged::page_index(pages, r.pos);
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
    const int heads = a.in[0].n + a.in[1].n + a.in[2].n;
    const long long task = (long long)blockIdx.x * ANY_WARPS + warp;
    if (task >= (long long)a.n_tokens * heads) return;
    const int t = (int)(task / heads);
    int h = (int)(task - (long long)t * heads);
    const int kind = h < a.in[0].n ? 0 : (h < a.in[0].n + a.in[1].n ? 1 : 2);
    const HeadsView& in = a.in[kind];
    const HeadsView& to = a.out[kind == 0 ? 0 : 1];
    h -= kind == 0 ? 0 : (kind == 1 ? a.in[0].n : a.in[0].n + a.in[1].n);

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
// Memory bounds it, and next to it the instructions: a block has heads of one kind (queries, keys or values), so that nothing but the numbers differs from
// head to head, and gain and angle are one set of coefficients per thread.  Blocks with all kinds needed 240 instructions per eight elements and 50 us for
// 8192 tokens of 40 heads of 128.  The loads of all of a thread's heads are requested first; while they are on their way the tokens'
// slots are looked up, a warp for each, and their angles turned.
// Threads of a block at most, and blocks per SM that the registers are held to (us, 8192 tokens of 40 heads / append of 4099 of 48): 384 x 3 39.5 / 26.7, 256 x 4 39.2 /
// 25.8, 128 x 8 37.0 / 25.3, 128 x 9 35.5 / 24.7, 128 x 10 36.5 / 25.4 (spills).
constexpr int ROPE_THREADS = 128;
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

struct RopePart {          // the blocks of one kind of head
    int32_t block0, heads, hb, per, tokens, ny;      // first block, heads, heads of a block and of a round, tokens of a block, blocks for the heads of a token
};
struct RopePlan {
    RopePart part[3];
};

template <typename T, int LH, bool APPEND, bool INTER>
__global__ void __launch_bounds__(ROPE_THREADS, 9) k_norm_rope(const __grid_constant__ NormRopeArgs a, const __grid_constant__ RopePlan plan) {
    constexpr int ROUNDS = ROPE_ROUNDS<T>, D = LH * 8;
    __shared__ __align__(16) float2 s_turn[ROPE_PAIRS];       // [token of the block][pair]
    __shared__ Slot s_slot[ROPE_TOKENS];
    const int kind = (int)blockIdx.x >= plan.part[2].block0 ? 2 : ((int)blockIdx.x >= plan.part[1].block0 ? 1 : 0);
    const RopePart part = plan.part[kind];
    const HeadsView in = a.in[kind];
    const int block = blockIdx.x - part.block0, by = block % part.ny, t0 = block / part.ny * part.tokens, n_tok = min(part.tokens, a.n_tokens - t0);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, l = tid % LH;
    const int tk = tid / (part.per * LH), hg = by * part.hb + (tid - tk * part.per * LH) / LH, h_end = min(by * part.hb + part.hb, part.heads), t = t0 + tk;
    const int n_here = tk < n_tok && hg < h_end ? (h_end - hg + part.per - 1) / part.per : 0;      // heads of this thread
    // the lane's two groups of four elements, and whether they are pairs that turn
    const int j = l * 4;
    const bool turns = j < a.pairs;
    const int o1 = INTER ? 2 * j : (turns ? j : a.pairs + j), o2 = INTER ? 2 * j + 4 : (turns ? a.pairs + j : D / 2 + j);
    Vec4<T> x1[ROUNDS], x2[ROUNDS];
    {
        const T* p = reinterpret_cast<const T*>(in.p) + paged::out_offset(in, t, hg);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r, p += part.per * in.head)
            if (r < n_here) {
                x1[r].load(p + o1);
                x2[r].load(p + o2);
            }
    }
    if (APPEND) {
        for (int k = warp; k < n_tok; k += blockDim.x >> 5) {
            const Slot slot = find_slot(a.seq, a.pages, t0 + k, lane);
            if (lane == 0) s_slot[k] = slot;
        }
        if (!a.positions || kind == 2) __syncthreads();       // the angles wait for the slots
    }
    const int kept = (a.pairs + 3) & ~3;
    if (!APPEND || kind < 2) {
        for (int i = tid; i < n_tok * kept; i += blockDim.x) {
            const int k = i / kept, pair = i - k * kept;
            if (pair < a.pairs) s_turn[i] = rope_turn(a.positions ? __ldg(a.positions + t0 + k) : s_slot[k].pos, __ldg(a.freq + pair), a.amplitude);
        }
        __syncthreads();
    }
    if (n_here == 0) return;                 // (whole groups of LH lanes)
    T* y;
    long long step;
    if (APPEND) {
        const Slot slot = s_slot[tk];
        if (slot.page < 0) return;
        if (kind) {
            y = reinterpret_cast<T*>(kind == 2 ? a.pages.v : a.pages.k) + (slot.page * a.pages.page + slot.slot * a.pages.tok + hg * a.pages.head);
            step = part.per * a.pages.head;
        }
    }
    if (!APPEND || kind == 0) {
        const HeadsView to = a.out[APPEND ? 0 : kind];
        y = reinterpret_cast<T*>(to.p) + paged::out_offset(to, t, hg);
        step = part.per * to.head;
    }
    if (APPEND && kind == 2) {               // values go as they are
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r, y += step)
            if (r < n_here) {
                x1[r].store(y + o1);
                x2[r].store(y + o2);
            }
        return;
    }
    // gain and angle as one: a pair (u, w) becomes root * (u * uc - w * ws, w * wc + u * us)
    const T* gain = reinterpret_cast<const T*>(kind ? a.k_gain : a.q_gain);
    float uc[4], us[4], wc[4], ws[4];
    {
        float f1[4] = {1.f, 1.f, 1.f, 1.f}, f2[4] = {1.f, 1.f, 1.f, 1.f};
        if (gain) {
            Vec4<T> g;
            g.load(gain + o1);
            g.get(f1);
            g.load(gain + o2);
            g.get(f2);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 cs = j + e < a.pairs ? s_turn[tk * kept + j + e] : make_float2(1.f, 0.f);
            // (interleaved: pair e is elements 2e and 2e + 1 of the eight)
            const float fu = INTER ? (e < 2 ? f1[2 * e & 3] : f2[2 * e & 3]) : f1[e], fw = INTER ? (e < 2 ? f1[(2 * e + 1) & 3] : f2[(2 * e + 1) & 3]) : f2[e];
            uc[e] = fu * cs.x; us[e] = fu * cs.y;
            wc[e] = fw * cs.x; ws[e] = fw * cs.y;
        }
    }
    const uint32_t group = LH == 32 ? 0xffffffffu : ((1u << LH) - 1u) << (lane & ~(LH - 1));      // the lanes of a head have the same rounds
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r, y += step) {
        if (r >= n_here) break;
        float u[4], w[4];
        x1[r].get(u);
        x2[r].get(w);
        float root = 1.f;
        if (gain) {
            float sq = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) sq = fmaf(w[e], w[e], fmaf(u[e], u[e], sq));
#pragma unroll
            for (int o = LH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(group, sq, o);
            root = rsqrtf(fmaf(sq, 1.f / D, a.eps));
        }
        // what does not turn has a sine of 0, but may be infinite: it is not multiplied by it
        if (INTER) {
            const float p[8] = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
            float q[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool turn = j + e < a.pairs;
                q[2 * e] = turn ? fmaf(p[2 * e], uc[e], -(p[2 * e + 1] * ws[e])) : p[2 * e] * uc[e];
                q[2 * e + 1] = turn ? fmaf(p[2 * e + 1], wc[e], p[2 * e] * us[e]) : p[2 * e + 1] * wc[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) { u[e] = q[e]; w[e] = q[4 + e]; }
        } else if (turns) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = u[e], z = w[e];
                u[e] = fmaf(x, uc[e], -(z * ws[e]));
                w[e] = fmaf(z, wc[e], x * us[e]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { u[e] *= uc[e]; w[e] *= wc[e]; }
        }
        if (gain) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { u[e] *= root; w[e] *= root; }
        }
        x1[r].set(u);
        x2[r].set(w);
        x1[r].store(y + o1);
        x2[r].store(y + o2);
    }
}

template <typename T, int LH>
int run_norm_rope(const NormRopeArgs& a, cudaStream_t s) {
    constexpr int ROUNDS = ROPE_ROUNDS<T>;
    const int all = a.in[0].n + a.in[1].n + a.in[2].n, most = 128 / LH, kept = (a.pairs + 3) & ~3;
    // a call that does not fill the GPU spreads its heads over the SMs, a head per thread group
    const bool small = (long long)a.n_tokens * ((all + most - 1) / most) <= 4 * 148;
    RopePlan plan;
    long long blocks = 0;
    int threads = 32;
    for (int kind = 0; kind < 3; ++kind) {
        RopePart& p = plan.part[kind];
        p.block0 = (int)blocks;
        p.heads = a.in[kind].n;
        p.hb = p.per = p.tokens = p.ny = 1;
        if (p.heads == 0) continue;
        if (small) {
            p.hb = p.per = p.heads < most ? p.heads : most;
        } else {
            const int cap = ROUNDS * (ROPE_THREADS / LH);
            p.ny = (p.heads + cap - 1) / cap;
            p.hb = (p.heads + p.ny - 1) / p.ny;
            p.per = (p.hb + ROUNDS - 1) / ROUNDS;
            // as many tokens as a block has threads for, but a block for every SM
            p.tokens = ROPE_THREADS / (p.per * LH);
            if (p.tokens > ROPE_TOKENS) p.tokens = ROPE_TOKENS;
            if (kept && p.tokens > ROPE_PAIRS / kept) p.tokens = ROPE_PAIRS / kept;
            if (p.tokens > a.n_tokens / 148) p.tokens = a.n_tokens / 148;
            if (p.tokens < 1) p.tokens = 1;
        }
        p.ny = (p.heads + p.hb - 1) / p.hb;
        const int need = (p.tokens * p.per * LH + 31) / 32 * 32;
        if (need > threads) threads = need;
        blocks += (long long)((a.n_tokens + p.tokens - 1) / p.tokens) * p.ny;
    }
    for (int kind = 1; kind < 3; ++kind)            // a kind that is not there has no blocks
        if (plan.part[kind].heads == 0) plan.part[kind].block0 = 0x7fffffff;
    if (blocks > 0x7ffffffe) return -1;
    const bool inter = a.pairs && a.interleaved;
    const unsigned grid = (unsigned)blocks;
    if (a.append) {
        if (inter) k_norm_rope<T, LH, true, true><<<grid, threads, 0, s>>>(a, plan);
        else k_norm_rope<T, LH, true, false><<<grid, threads, 0, s>>>(a, plan);
    } else {
        if (inter) k_norm_rope<T, LH, false, true><<<grid, threads, 0, s>>>(a, plan);
        else k_norm_rope<T, LH, false, false><<<grid, threads, 0, s>>>(a, plan);
    }
    return 0;
}
template <typename T>
int run_norm_rope_d(const NormRopeArgs& a, cudaStream_t s) {
    return a.D == 32 ? run_norm_rope<T, 4>(a, s) : (a.D == 64 ? run_norm_rope<T, 8>(a, s) : (a.D == 128 ? run_norm_rope<T, 16>(a, s) : run_norm_rope<T, 32>(a, s)));
}
bool fast_shape(const NormRopeArgs& a, int elem) {
    if (a.D != 32 && a.D != 64 && a.D != 128 && a.D != 256) return false;
    if (a.pairs && !a.interleaved && a.pairs % 4) return false;
    const int per16 = 16 / elem;
    auto al = [&](const HeadsView& v) { return !v.p || (reinterpret_cast<uintptr_t>(v.p) % 16 == 0 && v.tok % per16 == 0 && v.head % per16 == 0); };
    auto al_p = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
    if (!al(a.in[0]) || !al(a.in[1]) || !al(a.in[2]) || !al(a.out[0]) || !al(a.out[1]) || !al_p(a.q_gain) || !al_p(a.k_gain)) return false;
    return !a.append || (al_p(a.pages.k) && al_p(a.pages.v) && a.pages.page % per16 == 0 && a.pages.tok % per16 == 0 && a.pages.head % per16 == 0);
}

}  // namespace

void launch_rope_table(const uint64_t* freq, int pairs, uint64_t* table, cudaStream_t s) {
    RopeFreqs r;
    for (int i = 0; i < ESP_ROPE_MAX_DIM / 2; ++i) r.f[i] = i < pairs ? freq[i] : 0;
    k_rope_table_paged<<<1, ESP_ROPE_MAX_DIM / 2, 0, s>>>(r, pairs, table);
}

int launch_norm_rope(int dtype, const NormRopeArgs& a, cudaStream_t s) {
    const int heads = a.in[0].n + a.in[1].n + a.in[2].n;
    if (fast_shape(a, dtype == 0 ? 4 : 2)) return dtype == 0 ? run_norm_rope_d<float>(a, s) : run_norm_rope_d<__nv_bfloat16>(a, s);
    const long long tasks = (long long)a.n_tokens * heads;
    const long long blocks = (tasks + ANY_WARPS - 1) / ANY_WARPS;
    if (blocks > 0x7fffffff) return -1;
    if (dtype == 0) k_norm_rope_any<float><<<(unsigned)blocks, ANY_WARPS * 32, 0, s>>>(a);
    else k_norm_rope_any<__nv_bfloat16><<<(unsigned)blocks, ANY_WARPS * 32, 0, s>>>(a);
    return 0;
}

}  // namespace esp
