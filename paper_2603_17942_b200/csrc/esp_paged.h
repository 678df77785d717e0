// Operators over a paged key/value cache: what their kernels are given, and the launches behind the C entry points.
#pragma once

#include "esp_common.cuh"

namespace esp {

struct HeadsView {      // as esp_heads; p NULL: absent
    void* p;
    long long tok, head;
    int32_t n;
};

// Where token s of page p of head h lives: p * page + s * tok + h * head elements behind k and v.
struct PagesView {
    void *k, *v;
    long long page, tok, head;
    int32_t n_pages, page_size, page_shift;     // log2 of page_size, -1 if it is no power of two
};
// log2 of x, -1 if x is no power of two: what is divided by on the way to a kernel's first load is a shift where it can be
inline int shift_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return (1 << s) == x ? s : -1;
}

struct SeqTable {
    const int32_t *q_start, *kv_len, *table;
    int32_t batch, table_stride, max_new, n_tokens;
    int32_t kv_cap;     // positions a row of the table can hold
    int32_t* status;
};

struct NormRopeArgs {
    HeadsView in[3], out[2];     // queries, keys, values
    const void *q_gain, *k_gain;
    const uint64_t* freq;        // [pairs] fractions of a turn per position, 2^64 = one turn
    const int32_t* positions;    // NULL: the slot's position (append)
    int32_t n_tokens, D, pairs, interleaved;
    float eps, amplitude;
    PagesView pages;             // append: where k and v go
    SeqTable seq;
    int32_t append;
};

struct __align__(16) MergeDesc {        // a tile that several CTAs share
    int32_t token, pairs, head0;
    int32_t parts;        // 4 x CTAs that have a piece of it + 2 if each of them has two parts + the first one's slot; 0: no such tile
    int32_t first;        // the first of these CTAs
    int32_t pad[3];
};

struct PagedAttnArgs {
    HeadsView q, out;
    float* lse;
    PagesView pages;
    SeqTable seq;
    const unsigned long long* anc;
    int32_t Hq, Hkv, group, D, window;
    float scale_log2;
    int32_t rows, rows_shift;   // tokens of a tile: rows * group (token, head) pairs
    int32_t pairs;          // pairs of a tile's partial in the scratch
    int32_t n_cta;          // CTAs the work is dealt to
    int32_t min_units;      // fewer CTAs rather than fewer chunks than this for each
    int32_t vec;            // CUDA-core kernel: rows can be read four elements at a time
    int32_t out_vec;        // rows of out can be written four elements at a time
    MergeDesc* desc;        // [PAGED_MAX_CTAS][2] the split tiles that a CTA has the first piece of, and a later piece of
    float4* part_o;         // [n_cta][2][D / 4][pairs] split partials: weighted values, not divided by the sum
    float2* part_ml;        // [n_cta][2][pairs] their (maximum in the log2 domain, sum)
};

// Partials a launch may need at most: two tiles of 256 pairs for each of 148 SMs, or as much in smaller tiles.
constexpr int PAGED_MAX_PAIRS = 256;
constexpr int PAGED_MAX_SMS = 148;
constexpr int PAGED_MAX_CTAS = PAGED_MAX_SMS * 8;

int launch_norm_rope(int dtype, const NormRopeArgs& a, cudaStream_t s);
void launch_rope_table(const uint64_t* freq, int pairs, uint64_t* table, cudaStream_t s);
int launch_paged_simt(int dtype, PagedAttnArgs a, int n_sm, cudaStream_t s);
bool paged_tc_supported(int dtype, const PagedAttnArgs& a);
int launch_paged_tc(PagedAttnArgs a, int n_sm, cudaStream_t s);
bool paged_tma_pages(const PagedAttnArgs& a, int chunk, int* box_rows);      // boxes of *box_rows slots can be copied
bool paged_few_supported(int dtype, const PagedAttnArgs& a);
int launch_paged_few(PagedAttnArgs a, int n_sm, cudaStream_t s);
int launch_paged_merge_few(int dtype, const PagedAttnArgs& a, cudaStream_t s);   // tiles of at most 16 pairs
int launch_paged_merge(int dtype, const PagedAttnArgs& a, cudaStream_t s);

}  // namespace esp
