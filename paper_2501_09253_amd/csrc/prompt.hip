// Entry points of the prompt attention: argument checks and the choice of kernel.
#include "prompt.h"
#include <cmath>

using namespace pserve;

static int current_device(int* dev) {
    PS_CHECK_HIP(hipGetDevice(dev));
    return PSERVE_OK;
}

static int check_desc(const pserve_prompt_desc* d, const char* who) {
    PS_REQUIRE(d, "%s: desc is NULL", who);
    PS_REQUIRE(d->n > 0, "%s: need n > 0 sequences", who);
    PS_REQUIRE(d->dtype == PSERVE_F32 || d->dtype == PSERVE_BF16, "%s: unknown dtype %d", who, d->dtype);
    PS_REQUIRE(d->heads > 0 && d->kv_heads > 0 && d->heads % d->kv_heads == 0, "%s: %d heads over %d key/value heads", who, d->heads, d->kv_heads);
    PS_REQUIRE(d->heads <= 4096, "%s: more than 4096 heads", who);
    PS_REQUIRE(d->head_dim > 0 && d->head_dim % 16 == 0 && d->head_dim <= 128, "%s: head_dim %d is not a multiple of 16 up to 128", who, d->head_dim);
    PS_REQUIRE(std::isfinite(d->scale), "%s: the scale is not finite", who);
    PS_REQUIRE(d->q_tokens >= 0 && d->q_tokens <= INT32_MAX && d->max_q >= 0 && d->max_k >= 0, "%s: negative or too large sizes", who);
    return PSERVE_OK;
}

// strides and pointers of a [tokens][heads][head_dim] tensor: 16-byte rows; the rows of a tile are addressed in 32 bits
static int check_tensor(const pserve_prompt_desc* d, const void* p, const int64_t* stride, const char* name, const char* who) {
    const int64_t vn = 16 / (int64_t)dtype_size(d->dtype);
    PS_REQUIRE(((uintptr_t)p & 15) == 0, "%s: %s is not 16-byte aligned", who, name);
    for (int i = 0; i < 2; ++i)
        PS_REQUIRE(stride[i] >= 0 && stride[i] < (int64_t)1 << (i ? 40 : 24) && stride[i] % vn == 0,
                   "%s: stride %lld of %s is not a multiple of 16 bytes or too large", who, (long long)stride[i], name);
    return PSERVE_OK;
}

static PromptArgs prompt_args(const pserve_prompt_desc* d) {
    PromptArgs a{};
    a.q_tokens = d->q_tokens;
    a.q_row = d->q_stride[0]; a.q_head = d->q_stride[1];
    a.o_row = d->o_stride[0]; a.o_head = d->o_stride[1];
    a.n = d->n; a.H = d->heads; a.Hk = d->kv_heads; a.G = d->heads / d->kv_heads; a.D = d->head_dim;
    a.causal = d->causal != 0;
    a.scale2 = (float)((double)d->scale * 1.4426950408889634);
    return a;
}

// Rows of a tile and shares of its keys.
static void choose(const pserve_prompt_desc* d, PromptArgs& a, int src) {
    const int64_t max_q = d->max_q ? d->max_q : cdiv(d->q_tokens, d->n), 
                  keys = d->max_k ? d->max_k : src == SRC_PACKED ? cdiv(std::max<int64_t>(d->k_tokens, 0), d->n) : 1024;
    if (d->dtype == PSERVE_BF16 && max_q * a.G > 16) {
        a.rows = src == SRC_PACKED && prompt_slots(a, a.G, 256) * a.Hk >= 512 ? 256 : 128;
        a.splits = (int)std::max<int64_t>(1, std::min(512 / (prompt_slots(a, a.G, a.rows) * a.Hk), keys / 512));
        return;
    }
    a.rows = 16;
    a.splits = 1;
    const int64_t items = prompt_slots(a, a.G, 16) * a.Hk;
    if (keys <= 512 || items >= 768) {         // a tile is one unit, nothing to join
        a.unit = INT32_MAX;
        a.lead = 0;
        a.blocks = (int32_t)std::min<int64_t>(items, 1 << 23);
    } else {
        a.unit = 128;
        a.lead = 1;
        a.blocks = (int32_t)std::max<int64_t>(1, std::min<int64_t>(512, items * cdiv(keys, 128) / 2));
    }
}

static size_t part_bytes(const PromptArgs& a) {
    const size_t tile = (size_t)a.rows * ((a.D <= 64 ? 64 : 128) + 2) * sizeof(float);
    if (a.rows == 16) return a.unit == INT32_MAX ? 0 : 2 * (size_t)a.blocks * tile;
    return a.splits == 1 ? 0 : (size_t)prompt_slots(a, a.G, a.rows) * a.Hk * a.splits * tile;
}

static int run(const pserve_prompt_desc* d, PromptArgs& a, int src, void* workspace, size_t bytes, hipStream_t st, const char* who) {
    if (d->q_tokens == 0) return PSERVE_OK;
    choose(d, a, src);
    // (a launch has at most 2^32 threads)
    PS_REQUIRE(prompt_slots(a, a.G, a.rows) * a.Hk * std::max(a.splits, 16) < (1 << 24), "%s: too many tiles of rows", who);
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
    PS_TRY(check_tensor(desc, q, desc->q_stride, "q", who));
    PS_TRY(check_tensor(desc, k, desc->k_stride, "k", who));
    PS_TRY(check_tensor(desc, v, desc->v_stride, "v", who));
    PS_TRY(check_tensor(desc, o, desc->o_stride, "o", who));
    PromptArgs a = prompt_args(desc);
    a.Q = q; a.K = k; a.V = v; a.O = o;
    a.cu_q = cu_q; a.cu_k = cu_k;
    a.k_tokens = desc->k_tokens;
    a.k_row = desc->k_stride[0]; a.k_head = desc->k_stride[1];
    a.v_row = desc->v_stride[0]; a.v_head = desc->v_stride[1];
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
    PS_TRY(check_tensor(desc, q, desc->q_stride, "q", who));
    PS_TRY(check_tensor(desc, o, desc->o_stride, "o", who));
    PromptArgs a = prompt_args(desc);
    a.Q = q; a.O = o; a.cu_q = cu_q;
    a.k8 = store->k; a.v8 = store->v; a.k_scale = store->k_scale; a.v_scale = store->v_scale;
    a.key_len = key_len; a.table = table; a.max_pages = max_pages;
    while ((1 << a.page_shift) < page) ++a.page_shift;
    a.pages = (int32_t)(store->places >> a.page_shift);
    return run(desc, a, SRC_STORE, workspace, workspace_bytes, (hipStream_t)stream, who);
}

}  // extern "C"
