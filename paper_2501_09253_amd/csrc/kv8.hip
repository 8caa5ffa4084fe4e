// The 8-bit key/value store: writing and reading rows (pserve_kv8_*).
//
// Both passes are bound by memory: a group (a token's head) of D values is 2 D or 4 D bytes on one side, D + 4 on the other.
// A group is taken by LPG lanes of eight values each, so 16 bytes a lane on the wide side.
#include "kv8.h"
#include "quant8.h"

using namespace pserve;

namespace pserve {

struct Kv8Args {
    const void *k, *v;
    void *ko, *vo;
    int8_t *k8, *v8;
    float *ks, *vs;
    int32_t* owner;
    const int64_t* places_of;
    int64_t rows, places, k_row, k_head, v_row, v_head;
    int32_t heads, dim;
};

// Which row of the call a place gets: the last one.  Calls of few rows look through the rows behind their own; larger ones
// leave their number in `owner` in a launch of its own, and the writing launch, which finds it, sets the place back to -1.
constexpr int KV8_LOOK = 128;

__global__ void __launch_bounds__(256)
kv8_claim_kernel(Kv8Args a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.rows) return;
    const int64_t p = a.places_of[i];
    if (p >= 0 && p < a.places) atomicMax(a.owner + p, (int32_t)i);
}
__global__ void __launch_bounds__(256)
kv8_release_kernel(Kv8Args a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.rows) return;
    const int64_t p = a.places_of[i];
    if (p >= 0 && p < a.places) a.owner[p] = -1;
}

template <typename T, int LPG, bool CLAIMED>
__global__ void __launch_bounds__(256)
kv8_write_kernel(Kv8Args a) {
    const int64_t g = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPG;      // group: (row, head)
    const int l = threadIdx.x % LPG;
    const bool vals = blockIdx.y != 0;
    const bool in = g < a.rows * a.heads;
    const int64_t row = in ? g / a.heads : 0;
    const int head = in ? (int)(g - row * a.heads) : 0;
    const int64_t p = a.places_of[row];
    bool mine = in && p >= 0 && p < a.places;
    if (CLAIMED) {
        if (mine) mine = a.owner[p] == (int32_t)row;
    } else if (mine) {
        bool later = false;
        for (int64_t j = row + 1 + l; j < a.rows; j += LPG) later |= a.places_of[j] == p;
        mine = !later;
    }
    if (!CLAIMED) {
        int other = !mine;
#pragma unroll
        for (int x = 1; x < LPG; x <<= 1) other |= __shfl_xor(other, x);
        mine = !other;
    }
    float x[8] = {};
    const bool has = 8 * l < a.dim;
    if (mine && has) load8((vals ? (const T*)a.v + row * a.v_row + head * a.v_head : (const T*)a.k + row * a.k_row + head * a.k_head) + 8 * l, x);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs_bits(x[i]));
#pragma unroll
    for (int s = 1; s < LPG; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
    if (!mine) return;
    const Quant8 z(m);
    const int64_t at = p * a.heads + head;
    if (has) *reinterpret_cast<q8_u32x2*>((vals ? a.v8 : a.k8) + at * a.dim + 8 * l) = pack8(z, x);
    if (l == 0) (vals ? a.vs : a.ks)[at] = z.scale;
}

template <typename T, int LPG>
__global__ void __launch_bounds__(256)
kv8_read_kernel(Kv8Args a) {
    const int64_t g = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPG;
    const int l = threadIdx.x % LPG;
    const bool vals = blockIdx.y != 0;
    if (g >= a.rows * a.heads || 8 * l >= a.dim) return;
    const int64_t row = g / a.heads, p = a.places_of[row];
    const int head = (int)(g - row * a.heads);
    float x[8] = {};
    if (p >= 0 && p < a.places) {
        const int64_t at = p * a.heads + head;
        const q8_u32x2 w = *reinterpret_cast<const q8_u32x2*>((vals ? a.v8 : a.k8) + at * a.dim + 8 * l);
        const float s = (vals ? a.vs : a.ks)[at];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)(int8_t)(w[i / 4] >> (8 * (i % 4))) * s;
    }
    store8((vals ? (T*)a.vo : (T*)a.ko) + g * a.dim + 8 * l, x);
}

__global__ void __launch_bounds__(256)
kv8_fill_kernel(u32x4* p, int64_t n, uint32_t value) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = u32x4{value, value, value, value};
}
static int fill(void* p, size_t bytes, uint32_t value, hipStream_t st) {
    const int64_t n = cdiv((int64_t)bytes, 16);             // the allocations are rounded up to 256 bytes
    kv8_fill_kernel<<<(unsigned)std::min<int64_t>(cdiv(n, 256), 4096), 256, 0, st>>>((u32x4*)p, n, value);
    return check_launch("kv8_fill_kernel");
}

template <typename T, int LPG>
static int kv8_write_as(const Kv8Args& a, hipStream_t st) {
    const dim3 grid((unsigned)cdiv(a.rows * a.heads * LPG, 256), 2);
    const unsigned per_row = (unsigned)cdiv(a.rows, 256);
    if (a.rows <= KV8_LOOK) {
        kv8_write_kernel<T, LPG, false><<<grid, 256, 0, st>>>(a);
        return check_launch("kv8_write_kernel");
    }
    kv8_claim_kernel<<<per_row, 256, 0, st>>>(a);
    PS_TRY(check_launch("kv8_claim_kernel"));
    kv8_write_kernel<T, LPG, true><<<grid, 256, 0, st>>>(a);
    PS_TRY(check_launch("kv8_write_kernel"));
    kv8_release_kernel<<<per_row, 256, 0, st>>>(a);
    return check_launch("kv8_release_kernel");
}
template <typename T, int LPG>
static int kv8_read_as(const Kv8Args& a, hipStream_t st) {
    kv8_read_kernel<T, LPG><<<dim3((unsigned)cdiv(a.rows * a.heads * LPG, 256), 2), 256, 0, st>>>(a);
    return check_launch("kv8_read_kernel");
}

}  // namespace pserve

static int check_device(const pserve_kv8_t* s, const char* who) {
    int dev;
    PS_CHECK_HIP(hipGetDevice(&dev));
    PS_REQUIRE(dev == s->device, "%s: the store is on device %d, the current one is %d", who, s->device, dev);
    return PSERVE_OK;
}

// up to 16 threads a group, fewer than 2^32 in a launch: refused before the first launch, so that no claim is left behind
static int check_rows(const pserve_kv8_t* s, int64_t rows, const char* who) {
    PS_REQUIRE(rows >= 0 && rows < (1 << 28) && rows * s->heads < (1 << 28), "%s: %lld rows of %d heads", who, (long long)rows, s->heads);
    return PSERVE_OK;
}

static Kv8Args kv8_args(const pserve_kv8_t* s) {
    Kv8Args a{};
    a.k8 = s->k; a.v8 = s->v; a.ks = s->k_scale; a.vs = s->v_scale; a.owner = s->owner;
    a.places = s->places; a.heads = s->heads; a.dim = s->dim;
    return a;
}

extern "C" {

int pserve_kv8_create(int64_t places, int32_t kv_heads, int32_t head_dim, void* stream, pserve_kv8_t** out) {
    static const char who[] = "pserve_kv8_create";
    PS_REQUIRE(out, "%s: out is NULL", who);
    *out = nullptr;
    PS_REQUIRE(places > 0 && places <= INT32_MAX, "%s: %lld places", who, (long long)places);
    PS_REQUIRE(kv_heads > 0 && kv_heads <= 4096, "%s: %d heads", who, kv_heads);
    PS_REQUIRE(head_dim > 0 && head_dim % 16 == 0 && head_dim <= 128, "%s: head_dim %d is not a multiple of 16 up to 128", who, head_dim);
    return guarded(who, [&]() -> int {
        std::unique_ptr<pserve_kv8_t> s(new pserve_kv8_t());
        s->places = places; s->heads = kv_heads; s->dim = head_dim;
        PS_CHECK_HIP(hipGetDevice(&s->device));
        hipStream_t st = (hipStream_t)stream;
        auto make = [&](void** p, size_t bytes, uint32_t value) -> int {
            bytes = (bytes + 255) / 256 * 256;
            PS_TRY(s->pool.alloc(p, bytes));
            return fill(*p, bytes, value, st);
        };
        const size_t groups = (size_t)places * kv_heads;
        PS_TRY(make((void**)&s->k, groups * head_dim, 0));
        PS_TRY(make((void**)&s->v, groups * head_dim, 0));
        PS_TRY(make((void**)&s->k_scale, groups * sizeof(float), 0));
        PS_TRY(make((void**)&s->v_scale, groups * sizeof(float), 0));
        PS_TRY(make((void**)&s->owner, (size_t)places * sizeof(int32_t), 0xffffffffu));
        PS_CHECK_HIP(hipStreamSynchronize(st));             // later calls may come on other streams
        *out = s.release();
        return PSERVE_OK;
    });
}

void pserve_kv8_free(pserve_kv8_t* store) { delete store; }

int pserve_kv8_write(pserve_kv8_t* store, const void* k, const void* v, int dtype, const int64_t k_stride[2],
                     const int64_t v_stride[2], const int64_t* places, int64_t rows, void* stream) {
    static const char who[] = "pserve_kv8_write";
    PS_REQUIRE(store && k_stride && v_stride, "%s: NULL argument", who);
    PS_REQUIRE(dtype == PSERVE_F32 || dtype == PSERVE_BF16, "%s: unknown dtype %d", who, dtype);
    PS_TRY(check_rows(store, rows, who));
    if (rows == 0) return PSERVE_OK;
    PS_REQUIRE(k && v && places, "%s: NULL buffer", who);
    PS_TRY(check_device(store, who));
    PS_REQUIRE(!(((uintptr_t)k | (uintptr_t)v) & 15), "%s: k and v must be 16-byte aligned", who);
    const int64_t vn = 16 / (int64_t)dtype_size(dtype);
    for (int i = 0; i < 2; ++i)                             // (that of a dimension of one is any number)
        PS_REQUIRE((i ? store->heads : rows) == 1 || (k_stride[i] >= 0 && v_stride[i] >= 0 && k_stride[i] % vn == 0 && v_stride[i] % vn == 0),
                   "%s: strides must be multiples of 16 bytes", who);
    Kv8Args a = kv8_args(store);
    a.k = k; a.v = v; a.places_of = places; a.rows = rows;
    a.k_row = k_stride[0]; a.k_head = k_stride[1]; a.v_row = v_stride[0]; a.v_head = v_stride[1];
    hipStream_t st = (hipStream_t)stream;
    if (dtype == PSERVE_BF16) return store->dim <= 64 ? kv8_write_as<uint16_t, 8>(a, st) : kv8_write_as<uint16_t, 16>(a, st);
    return store->dim <= 64 ? kv8_write_as<float, 8>(a, st) : kv8_write_as<float, 16>(a, st);
}

int pserve_kv8_read(const pserve_kv8_t* store, const int64_t* places, int64_t rows, int dtype, void* k, void* v, void* stream) {
    static const char who[] = "pserve_kv8_read";
    PS_REQUIRE(store, "%s: NULL argument", who);
    PS_REQUIRE(dtype == PSERVE_F32 || dtype == PSERVE_BF16, "%s: unknown dtype %d", who, dtype);
    PS_TRY(check_rows(store, rows, who));
    if (rows == 0) return PSERVE_OK;
    PS_REQUIRE(k && v && places, "%s: NULL buffer", who);
    PS_TRY(check_device(store, who));
    PS_REQUIRE(!(((uintptr_t)k | (uintptr_t)v) & 15), "%s: k and v must be 16-byte aligned", who);
    Kv8Args a = kv8_args(store);
    a.ko = k; a.vo = v; a.places_of = places; a.rows = rows;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == PSERVE_BF16) return store->dim <= 64 ? kv8_read_as<uint16_t, 8>(a, st) : kv8_read_as<uint16_t, 16>(a, st);
    return store->dim <= 64 ? kv8_read_as<float, 8>(a, st) : kv8_read_as<float, 16>(a, st);
}

}  // extern "C"
