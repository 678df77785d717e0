"""How the weights of cached positions count their work (no GPU): the host-side compilation of the counting functions against the definition, chunk by chunk and token by token."""
import subprocess

from paper_2603_17942_b200 import build as esp_build

PROGRAM = r"""
#include <stdio.h>
#include <string.h>
#include "esp_key_weights.cuh"

using namespace esp;
using namespace esp::paged;

static long long n_cases = 0, n_bad = 0;

template <int CK>
static void one(int n, int kv, int last, int rows, int window, bool tree) {
    static const unsigned long long masks[2] = {0, 0};
    KeyWeightArgs w;
    memset(&w, 0, sizeof(w));
    w.a.rows = rows;
    w.a.rows_shift = shift_of(rows);
    w.a.window = window;
    w.a.anc = tree ? masks : nullptr;
    w.last = last;
    Seq s;
    s.start = 0; s.n = n; s.kv = kv;
    const WSeq x = observed(w, s);
    const int i0 = last > 0 && n > last ? n - last : 0, T = (n - i0 + rows - 1) / rows, C = T > 0 ? (kv + CK - 1) / CK : 0;
    unsigned long long want = 0, by_chunk = 0;
    for (int c = 0; c < C; ++c) {
        int first = -1, end = 0;                          // tiles of which some token sees some key of the chunk
        for (int t = 0; t < T; ++t) {
            bool meets = tree;
            for (int i = i0 + t * rows; i < n && i < i0 + (t + 1) * rows && !meets; ++i) {
                const int P = kv - n + i, lo = window > 0 && P - window + 1 > 0 ? P - window + 1 : 0, p1 = (c + 1) * CK < kv ? (c + 1) * CK : kv;
                meets = P >= 0 && lo < p1 && P >= c * CK;
            }
            if (meets) { first = first < 0 ? t : first; end = t + 1; }
        }
        want += first < 0 ? 1 : end - first;
        const WChunk k = make_chunk<CK>(w, x, c);
        by_chunk += k.units();
        if (first >= 0 ? k.t0 != first || k.nt != end - first : k.nt != 0) want = ~0ull;
    }
    uint32_t got = 0;
    const bool counted = lane_units<CK>(w, x, got);
    ++n_cases;
    if (x.i0 != i0 || x.T != T || n_chunks<CK>(x) != C || by_chunk != want || (counted ? got != want : got != 0)) {
        if (++n_bad <= 20) printf("CK %d rows %d n %d kv %d last %d window %d tree %d: %llu units, by chunks %llu, counted %u\n", CK, rows, n, kv, last, window, tree, want, by_chunk, got);
    }
}

template <int CK>
static void all(int rows) {
    const int ns[] = {0, 1, 2, 7, 33, 128, 200, 205, 300, 543, 600, 807, 1500, 2000, 3000}, lasts[] = {0, 1, 40, 700, 5000};
    for (int n : ns) {
        const int kvs[] = {0, 1, 2, 10, 63, 64, 65, 234, 256, 257, 300, 700, 2000, n / 2, n - 600, n - 543, n - 300, n - 135, n - rows, n - 1, n, n + 1, n + 63, n + 400, n + 5000};
        for (int kv : kvs)
            if (kv >= 0)
                for (int last : lasts) {
                    one<CK>(n, kv, last, rows, 0, false);
                    one<CK>(n, kv, last, rows, 1, false);
                    one<CK>(n, kv, last, rows, 100, false);
                    if (n <= 128) one<CK>(n, kv, last, rows, 0, true);
                }
    }
}

int main() {
    for (int rows : {32, 18, 2, 128}) all<256>(rows);     // 128 pairs for groups of 4, 7, 64 and 1
    for (int rows : {8, 32, 5, 1}) all<64>(rows);         // 32 pairs for groups of 4, 1, 6 and 32
    for (int rows : {1, 7, 60, 3000}) all<32>(rows);
    printf("%lld cases, %lld wrong\n", n_cases, n_bad);
    return n_bad != 0;
}
"""

BOUNDS = r"""
#include <stdio.h>
#include <string.h>
#include "esp_key_weights.cuh"

using namespace esp;
using namespace esp::paged;

int main() {
    const long long most = 0x7fffffff;
    for (long long near : {1ll, 2ll, 3ll, 64ll, 1000ll, 1ll << 29, 1ll << 30, most})
        for (long long x = near - 1; x <= near + 1 && x <= most; ++x) {
            int want = -1;
            for (int s = 0; s < 31; ++s)
                if (x == 1ll << s) want = s;
            if (x > 0 && shift_of((int)x) != want) { printf("shift_of(%lld) is %d\n", x, shift_of((int)x)); return 1; }
        }
    // all observed tokens of any sequence are one tile, whatever bound the caller gives
    for (int tokens : {1, 60, 1 << 30})
        for (int max_new : {tokens, 100, (1 << 30) + 1, 0x7fffffff})
            for (int last : {0, 1, 40, 0x7fffffff}) {
                KeyWeightArgs w;
                memset(&w, 0, sizeof(w));
                w.a.seq.n_tokens = tokens;
                w.a.seq.max_new = max_new;
                w.last = last;
                w.a.rows = one_tile(w);
                w.a.rows_shift = shift_of(w.a.rows);
                for (int n : {0, 1, 2, 59, 60, 100, 1 << 30}) {
                    if (n > tokens || n > max_new) continue;
                    Seq s;
                    s.start = 0; s.n = s.kv = n;
                    const WSeq x = observed(w, s);
                    if (x.T != (n > 0) || w.a.rows < 1) { printf("tokens %d max_new %d last %d n %d: %d tiles of %d\n", tokens, max_new, last, n, x.T, w.a.rows); return 1; }
                }
            }
    return 0;
}
"""


def _compile(source, at):
    src, exe = str(at / "units.cu"), str(at / "units")
    with open(src, "w") as f:
        f.write(source)
    subprocess.run([esp_build.NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-I", esp_build.CSRC, "-o", exe, src], check=True, capture_output=True, text=True)
    return exe


def test_units_of_every_sequence(tmp_path):
    """Single tokens, prompts, observed tails, windows and trees; as many positions as tokens, more, fewer (padding), a few of them only and none."""
    done = subprocess.run([_compile(PROGRAM, tmp_path)], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stdout


def test_bounds_far_above_the_tokens(tmp_path):
    """max_new is a bound: 2^31 - 1 is one too.  (A power of two that was looked for beyond 2^30 was never found.)"""
    done = subprocess.run([_compile(BOUNDS, tmp_path)], capture_output=True, text=True, timeout=20)
    assert done.returncode == 0, done.stdout
