// Entry points of the prompt attention: argument checks and the choice of kernel.
#include "prompt.h"
#include <cmath>

using namespace pserve;

static int current_device(int* dev) {
    PS_CHECK_HIP(hipGetDevice(dev));
    return PSERVE_OK;
}

static float scale_log2(const pserve_prompt_desc* d) { return (float)((double)d->scale * 1.4426950408889634); }

static int check_desc(const pserve_prompt_desc* d, const char* who) {
    PS_REQUIRE(d, "%s: desc is NULL", who);
    PS_REQUIRE(d->n > 0, "%s: need n > 0 sequences", who);
    PS_REQUIRE(d->dtype == PSERVE_F32 || d->dtype == PSERVE_BF16, "%s: unknown dtype %d", who, d->dtype);
    PS_REQUIRE(d->heads > 0 && d->kv_heads > 0 && d->heads % d->kv_heads == 0, "%s: %d heads over %d key/value heads", who, d->heads, d->kv_heads);
    PS_REQUIRE(d->heads <= 4096, "%s: more than 4096 heads", who);
    PS_REQUIRE(d->head_dim > 0 && d->head_dim % 16 == 0 && d->head_dim <= 128, "%s: head_dim %d is not a multiple of 16 up to 128", who, d->head_dim);
    PS_REQUIRE(std::isfinite(d->scale) && std::isfinite(scale_log2(d)), "%s: the scale is not finite (or times log2(e) is not)", who);
    PS_REQUIRE(d->q_tokens >= 0 && d->q_tokens <= INT32_MAX && d->max_q >= 0 && d->max_k >= 0, "%s: negative or too large sizes", who);
    return PSERVE_OK;
}

// strides and pointers of a [tokens][heads][head_dim] tensor: 16-byte rows; the rows of a tile are addressed in 32 bits.  The stride of a
// dimension of one (or none) is any number: it counts as 0.
static int check_tensor(const pserve_prompt_desc* d, const void* p, const int64_t* stride, int64_t tokens, int32_t heads, const char* name, const char* who,
                        int64_t& row, int64_t& head) {
    const int64_t vn = 16 / (int64_t)dtype_size(d->dtype);
    PS_REQUIRE(((uintptr_t)p & 15) == 0, "%s: %s is not 16-byte aligned", who, name);
    row = tokens > 1 ? stride[0] : 0;
    head = heads > 1 ? stride[1] : 0;
    PS_REQUIRE(row >= 0 && row < (int64_t)1 << 24 && row % vn == 0 && head >= 0 && head < (int64_t)1 << 40 && head % vn == 0,
               "%s: a stride of %s (%lld, %lld) is not a multiple of 16 bytes or too large", who, name, (long long)row, (long long)head);
    return PSERVE_OK;
}

static PromptArgs prompt_args(const pserve_prompt_desc* d) {
    PromptArgs a{};
    a.q_tokens = d->q_tokens;
    a.n = d->n; a.Hk = d->kv_heads; a.G = d->heads / d->kv_heads; a.D = d->head_dim;
    a.causal = d->causal != 0;
    a.scale2 = scale_log2(d);
    return a;
}

// Rows of a tile, and shares of its keys where the call has few tiles: a tile of 16 rows needs the least work for few rows, one of 256 reads
// and turns its keys for the most rows but needs the whole register file.  us measured for 16 / 128 / 256 rows, the last two with their best
// number of shares (bf16, packed; "n of queries x keys", 8 heads of keys with 4 of queries each; heads of 64, then of 128 values):
//   1 of 256 x 256       9 / 11 / 15      12 / 15 / 23          2 of 1024 x 1024     64 / 37 / 28     124 / 51 / 45
//   32 of 8 x 2048      32 / 50 / 46      61 / 72 / 76          1 of 512 x 4096      86 / 48 / 38     154 / 81 / 57
//   8 of 77 x 77        14 /  8 / 12      22 / 11 / 18          32 of 512 x 512     352 / 115 / 88    730 / 271 / 236
//   8 of 300 x 300      48 / 21 / 21      94 / 39 / 43          1 of 8192 x 8192   1184 / 486 / 277  2445 / 1038 / 516
// and with 12 heads, each with its own keys:
//   32 of 8 x 2048      43 / 64 / 67      96 / 133 / 135        32 of 512 x 512     140 / 57 / 62     274 / 121 / 135
//   8 of 77 x 77         8 /  8 / 12      10 / 11 / 20          1 of 8192 x 8192    453 / 201 / 152   930 / 435 / 234
// and where 16 rows meet 128, n of queries x keys in 16 / 128 rows (heads of 64, then of 128):
//   12 heads:    16 of 24 x 1200   28 / 33    41 / 47       16 of 33 x 1200   43 / 33    75 / 47       4 of 64 x 4000   33 / 30    51 / 47
//                 8 of 24 x 600    18 / 19    25 / 24        8 of 40 x 600    22 / 19    32 / 26      32 of 40 x 700    32 / 30    59 / 60
//   4 x 8 heads: 16 of 8 x 1200    23 / 26    33 / 39       16 of 9 x 1200    35 / 26    53 / 40       4 of 16 x 4000   26 / 23    39 / 35
// So: 16 rows for sequences of up to 32 rows and where there are few tiles with few keys; 256 where they are filled, the mask's diagonal is
// a small part of them (keys * G) and they keep the chip busy; else 128.  Over the 8-bit store, whose keys are turned into bf16 on their way
// to the matrix cores, there is no form of 256 rows.
static void choose(const pserve_prompt_desc* d, PromptArgs& a, int src) {
    const int64_t max_q = d->max_q ? d->max_q : cdiv(d->q_tokens, d->n),
                  mean = src == SRC_PACKED ? cdiv(std::min<int64_t>(std::max<int64_t>(d->k_tokens, 1), 1 << 30), d->n) : 1024,
                  keys = src == SRC_PACKED && d->k_tokens == 0 ? 0 : d->max_k ? d->max_k : mean;       // (no packed keys: nothing to cut)
    auto tiles = [&](int rows) { return prompt_slots(a, a.G, rows) * a.Hk; };
    a.splits = 1;
    if (d->dtype == PSERVE_BF16 && max_q * a.G > 32 && (keys > 512 || tiles(16) >= 768)) {
        const bool wide = src == SRC_PACKED && max_q * a.G >= 256 && keys * a.G >= 1024 && tiles(256) * keys >= (1 << 18);
        a.rows = wide ? 256 : 128;
        // Shares of the keys fill the chip, with one block a CU or two: 1 of 512 x 4096, 12 heads, in 240 / 480 / 720 blocks takes 34 / 32 / 36 us
        // packed with heads of 64, 47 / 56 / 65 with heads of 128; over the store 49 / 40 / 45 and 59 / 50 / 58 (8 x 4 heads in 272 / 544 /
        // 816: 84 / 62 / 75 and 99 / 80 / 96).  Where the longest sequence has more keys than the mean most blocks end early, so more are
        // wanted: 8 of 32 x 100 .. 12800, 8 x 4 heads of 128: 201 us in 256, 85 in 768.  (Of the store only the longest is known: there the
        // same call takes 145 us in 512 where 64 is possible in 2048.)  Joining the shares has its price: 4 of 20 .. 700 (8 x 4 heads of 64)
        // take 21 us in one share, 32 in two; 2 of 1024 x 1024 (12 heads of 64) 28 and 32.
        int64_t want = wide || (src == SRC_PACKED && a.D > 64) ? 256 : 512;
        const int64_t t = tiles(a.rows);
        if (src == SRC_PACKED) want = want * std::min(std::max(keys, mean), 3 * mean) / mean;
        if (4 * t < 3 * want && 7 * t <= want * keys / 512) a.splits = (int)std::max<int64_t>(1, std::min(cdiv(want, t), keys / (wide ? 512 : 256)));
        return;
    }
    a.rows = 16;
    const int64_t items = tiles(16);
    // up to 512 keys a block has a tile to itself: cutting it costs more than it saves; so it is where there are tiles enough
    if (keys <= 512 || items >= 768) {
        a.unit = a.lead = 0;
        a.items = (int32_t)std::min<int64_t>(items, INT32_MAX);     // (more are refused)
        a.blocks = (int32_t)std::min<int64_t>(items, 1 << 23);
    } else {
        a.unit = 128;
        a.lead = 1;                             // (32 tokens over 12 .. 8000 keys of the store: 45 us with none, 37, 38, 39 with 1, 2, 3)
        a.blocks = (int32_t)std::max<int64_t>(1, std::min<int64_t>(512, items * cdiv(keys, 128) / 2));
    }
}

static size_t part_bytes(const PromptArgs& a) {
    const size_t tile = (size_t)a.rows * ((a.D <= 64 ? 64 : 128) + 2) * sizeof(float);
    if (a.rows == 16) return a.unit == 0 ? 0 : 2 * (size_t)a.blocks * tile;
    return a.splits == 1 ? 0 : (size_t)prompt_slots(a, a.G, a.rows) * a.Hk * a.splits * tile;
}

static int run(const pserve_prompt_desc* d, PromptArgs& a, int src, void* workspace, size_t bytes, hipStream_t st, const char* who) {
    if (d->q_tokens == 0) return PSERVE_OK;
    choose(d, a, src);
    // (a launch has fewer than 2^32 threads; the blocks of the 16-row tiles share them out, numbered in 31 bits)
    const int64_t tiles = prompt_slots(a, a.G, a.rows) * a.Hk;
    PS_REQUIRE(a.rows == 16 ? tiles <= INT32_MAX : tiles * std::max(a.splits, a.rows / 16) < (1 << 24), "%s: too many tiles of rows", who);
    const size_t need = part_bytes(a);
    PS_REQUIRE(bytes >= need && (need == 0 || (workspace && ((uintptr_t)workspace & 15) == 0)), "%s: workspace of %zu bytes, %zu needed (16-byte aligned)", who,
               bytes, need);
    a.part = (float*)workspace;
    return a.rows == 16 ? launch_prompt_few(a, d->dtype, src, st) : launch_prompt_tile(a, a.rows, src, st);
}

extern "C" {

int pserve_prompt_attention_workspace(const pserve_prompt_desc* desc, size_t* bytes) {
    PS_REQUIRE(bytes, "pserve_prompt_attention_workspace: NULL argument");
    PS_TRY(check_desc(desc, "pserve_prompt_attention_workspace"));
    PromptArgs a = prompt_args(desc);
    size_t need[2];                             // of pserve_prompt_attention and of pserve_kv8_attention
    for (int src : {SRC_PACKED, SRC_STORE}) {
        choose(desc, a, src);
        need[src] = part_bytes(a);
    }
    *bytes = std::max(need[0], need[1]);
    return PSERVE_OK;
}

int pserve_prompt_attention(const pserve_prompt_desc* desc, const void* q, const void* k, const void* v, const int32_t* cu_q,
                            const int32_t* cu_k, void* workspace, size_t workspace_bytes, void* o, void* stream) {
    static const char who[] = "pserve_prompt_attention";
    PS_TRY(check_desc(desc, who));
    PS_REQUIRE(desc->k_tokens >= 0 && desc->k_tokens <= (1 << 30), "%s: negative or too large sizes", who);
    if (desc->q_tokens == 0) return PSERVE_OK;
    PS_REQUIRE(q && o && cu_q && cu_k && ((k && v) || desc->k_tokens == 0), "%s: NULL buffer", who);
    PromptArgs a = prompt_args(desc);
    PS_TRY(check_tensor(desc, q, desc->q_stride, desc->q_tokens, desc->heads, "q", who, a.q_row, a.q_head));
    PS_TRY(check_tensor(desc, k, desc->k_stride, desc->k_tokens, desc->kv_heads, "k", who, a.k_row, a.k_head));
    PS_TRY(check_tensor(desc, v, desc->v_stride, desc->k_tokens, desc->kv_heads, "v", who, a.v_row, a.v_head));
    PS_TRY(check_tensor(desc, o, desc->o_stride, desc->q_tokens, desc->heads, "o", who, a.o_row, a.o_head));
    a.Q = q; a.K = k; a.V = v; a.O = o;
    a.cu_q = cu_q; a.cu_k = cu_k;
    a.k_tokens = desc->k_tokens;
    return run(desc, a, SRC_PACKED, workspace, workspace_bytes, (hipStream_t)stream, who);
}

int pserve_kv8_attention(const pserve_kv8_t* store, const pserve_prompt_desc* desc, const void* q, const int32_t* cu_q,
                         const int32_t* key_len, const int32_t* table, int32_t max_pages, int32_t page, void* workspace,
                         size_t workspace_bytes, void* o, void* stream) {
    static const char who[] = "pserve_kv8_attention";
    PS_REQUIRE(store, "%s: store is NULL", who);
    PS_TRY(check_desc(desc, who));
    PS_REQUIRE(desc->kv_heads == store->heads && desc->head_dim == store->dim, "%s: the store has %d heads of %d values", who, store->heads, store->dim);
    PS_REQUIRE(page > 0 && (page & (page - 1)) == 0, "%s: page %d is no power of two", who, page);
    PS_REQUIRE(max_pages >= 0 && (int64_t)max_pages * page <= (1 << 30), "%s: %d pages of %d tokens", who, max_pages, page);
    if (desc->q_tokens == 0) return PSERVE_OK;
    PS_REQUIRE(q && o && cu_q && key_len && (table || max_pages == 0), "%s: NULL buffer", who);
    int dev;
    PS_TRY(current_device(&dev));
    PS_REQUIRE(dev == store->device, "%s: the store is on device %d, the current one is %d", who, store->device, dev);
    PromptArgs a = prompt_args(desc);
    PS_TRY(check_tensor(desc, q, desc->q_stride, desc->q_tokens, desc->heads, "q", who, a.q_row, a.q_head));
    PS_TRY(check_tensor(desc, o, desc->o_stride, desc->q_tokens, desc->heads, "o", who, a.o_row, a.o_head));
    a.Q = q; a.O = o; a.cu_q = cu_q;
    a.k8 = store->k; a.v8 = store->v; a.k_scale = store->k_scale; a.v_scale = store->v_scale;
    a.key_len = key_len; a.table = table; a.max_pages = max_pages;
    while ((1 << a.page_shift) < page) ++a.page_shift;
    a.places = (uint32_t)store->places;
    a.pages = (uint32_t)cdiv(store->places, page);
    return run(desc, a, SRC_STORE, workspace, workspace_bytes, (hipStream_t)stream, who);
}

}  // extern "C"
