// Operators over a paged key/value cache: what their kernels are given, and the launches behind the C entry points.
#pragma once

#include <cuda.h>

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
    while (s < 30 && (1 << s) < x) ++s;         // (2^30 is the largest there is)
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

// Where the 32-bit number of token s of page p of head h is: p * page + s * tok + h * head elements behind p; NULL: absent
struct SlotsView {
    void* p;
    long long page, tok, head;
};

// Weights of cached positions (esp_paged_key_weights).  a: queries, pages, sequences, masks and the deal, as in the attention; rows = tokens of a tile.
struct KeyWeightArgs {
    PagedAttnArgs a;
    const float* lse;       // [n_tokens][Hq]
    SlotsView scores;
    int32_t last;           // observed tokens of a sequence at most (0: all)
    float keep;
    float* part;            // [n_cta][2][keys of a chunk] sums of the pieces of chunks that several CTAs share
};

// Blocks for a list of eviction: as many as hold the keys of the longest one that the table has room for, up to EVICT_BLOCKS.  Where that is more than the GPU takes at a time, blocks that a
// short list does not need cost it (barriers, and the moves within the first kernel), and rows of a table are often as long as the longest context: then it goes by what the scratch is
// made for, and each list that fits into one block has one (`as_needed`).  us, 256 lists of 2049 keys and 128 of 8000, cut to 2048 and 1000, with 1, 2, 4 and 8 blocks: 19, 33, 64,
// 139 and 51, 51, 59, 82; where the GPU is not full, others read a list sooner: 32 of 8000 27, 24, 22, 24.
constexpr int EVICT_KEYS = 8192, EVICT_BLOCKS = 8;        // keys that a block keeps, blocks of a cluster at most
inline int evict_blocks(int kv_cap, int list_cap, int lists, int n_sm, int32_t* as_needed) {
    auto holding = [](long long keys) {
        int n = 1;
        while (n < EVICT_BLOCKS && keys > (long long)n * EVICT_KEYS) n *= 2;
        return n;
    };
    const int n = holding(kv_cap);
    *as_needed = (long long)lists * n > 2ll * n_sm;
    return *as_needed ? holding(2ll * list_cap < kv_cap ? 2ll * list_cap : kv_cap) : n;
}

struct EvictArgs {
    PagesView pages;
    SlotsView scores, positions;
    SeqTable seq;           // (q_start is not read)
    const int32_t *seen, *budget;
    int32_t *settled, *kv_out;
    int32_t recent, Hkv, D;
    int32_t list_cap;       // moves of a list at most
    int32_t vec;            // elements of a row that can be moved at a time
    int32_t as_needed;      // a list whose keys fit into one block has one, whatever the others of the call need
    int32_t* count;         // [batch * Hkv] moves
    int4* info;             // [batch] (kv_len from now on, -1: as it was; settled slots and their positions' base as the call found them)
    int2* list;             // [batch * Hkv][list_cap] (from, to)
};

struct AcceptArgs {
    PagesView pages;
    SeqTable seq;
    const int32_t *parents, *drafted, *chosen;
    int32_t *tokens_out, *rows_out, *n_out, *kv_out;
    int32_t out_stride, Hkv, D, vec;
};

constexpr int SAMPLE_SLICE = 8192, SAMPLE_CAP = 160, SAMPLE_MAX_SLICES = 256, SAMPLE_BINS = 512;
// Weights are added up in 32-bit counters in 1 / unit of the most that one of them can be: the unit for a counter that `elements` may be added to.
constexpr unsigned SAMPLE_UNIT = 32768;
__host__ __device__ constexpr unsigned sample_unit(unsigned elements) { return 0xffffffffu / elements < SAMPLE_UNIT ? 0xffffffffu / elements : SAMPLE_UNIT; }
struct SampleSlice {        // what the first pass leaves of a slice of a row
    unsigned long long best;          // its first element in the order
    float cut;                        // its elements that are not below this are in its list (infinity: it has none)
    int32_t n;                        // elements of the list
    double stretch[8];                // sums of weights of its eighths, in terms of its own largest
};
struct SampleRest {
    double S;               // the row's weights, where top-p goes by them
    float M;                // its largest logit
    int32_t row;
};
struct SampleArgs {
    const void* logits;
    long long row_stride;
    int32_t n_rows, vocab;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t* top_k;
    int32_t* tokens;
    float* logprob;
    int32_t chunk;          // logits of a row that each block of its cluster has (the rest)
    int32_t slices;         // of a row
    float unit, per_unit;   // of the rest's histograms of weights (sample_unit), and its inverse
    SampleSlice* slice;     // [n_rows][slices]
    unsigned long long* entries;      // [n_rows][slices][SAMPLE_CAP]
    SampleRest* rest;       // rows that the lists do not settle
    int32_t* n_rest;
};

// Partials a launch may need at most: two tiles of 256 pairs for each of 148 SMs, or as much in smaller tiles.
constexpr int PAGED_MAX_PAIRS = 256;
constexpr int PAGED_MAX_SMS = 148;
constexpr int PAGED_MAX_CTAS = PAGED_MAX_SMS * 8;
constexpr int KEY_WEIGHT_KEYS = 256;      // keys of a chunk of the weights' kernels at most

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
int paged_page_map5(CUtensorMap* map, const PagedAttnArgs& a, const void* base, int box_rows);      // [pages][heads][halves][slots][64], box 64 x box_rows x halves
int paged_page_map(CUtensorMap* map, const PagedAttnArgs& a, const void* base, int box_rows);       // [pages][heads][slots][D], box 64 x box_rows
int launch_key_weights_join(const KeyWeightArgs& w, int keys, cudaStream_t s);
bool key_weights_few_supported(int dtype, const KeyWeightArgs& w);      // a handful of pairs
bool key_weights_rows_supported(int dtype, const KeyWeightArgs& w);     // any number of them
int launch_key_weights_few(KeyWeightArgs w, int n_sm, cudaStream_t s);
bool key_weights_tc_supported(int dtype, const KeyWeightArgs& w);
int launch_key_weights_tc(KeyWeightArgs w, int n_sm, cudaStream_t s);
int launch_key_weights_simt(int dtype, KeyWeightArgs w, int n_sm, cudaStream_t s);
int launch_evict(int dtype, const EvictArgs& a, int n_sm, cudaStream_t s);
int launch_accept(int dtype, const AcceptArgs& a, cudaStream_t s);
int launch_sample(int dtype, SampleArgs a, int n_sm, cudaStream_t s);

}  // namespace esp
