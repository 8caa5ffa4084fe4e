// The 8-bit key/value store: writing and reading rows (pserve_kv8_*).
//
// Both passes move a group (a token's head) of D values as 2 D or 4 D bytes on one side and D + 4 on the other.  A group is taken by LPG
// lanes of eight values each, so 16 bytes a lane on the wide side.  20,011 tokens of 8 heads of 128, bf16 (125 MB each way): reading
// 22 us, writing 37 with the claim.
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
// leave their number in `owner` in a launch of its own.  In the writing launch a block has whole rows: the row that finds its own number
// sets the place back to -1 once the block has looked, and a row that looks later finds -1, which is not its number either.
constexpr int KV8_LOOK = 128;

__global__ void __launch_bounds__(256)
kv8_claim_kernel(Kv8Args a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.rows) return;
    const int64_t p = a.places_of[i];
    if (p >= 0 && p < a.places) atomicMax(a.owner + p, (int32_t)i);
}
template <typename T, int LPG>
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
    if (mine) {
        bool later = false;
        for (int64_t j = row + 1 + l; j < a.rows; j += LPG) later |= a.places_of[j] == p;
        mine = !later;
    }
    int other = !mine;
#pragma unroll
    for (int x = 1; x < LPG; x <<= 1) other |= __shfl_xor(other, x);
    mine = !other;
    Raw8<T> raw = {};
    const bool has = 8 * l < a.dim;
    if (mine && has) load_raw((vals ? (const T*)a.v + row * a.v_row + head * a.v_head : (const T*)a.k + row * a.k_row + head * a.k_head) + 8 * l, raw);
    const uint32_t m = lanes_max<LPG>(largest8(0, raw));
    if (!mine) return;
    float x[8];
    values8(raw, x);
    const Quant8 z(m);
    const int64_t at = p * a.heads + head;
    if (has) *reinterpret_cast<q8_u32x2*>((vals ? a.v8 : a.k8) + at * a.dim + 8 * l) = pack8(z, x);
    if (l == 0) (vals ? a.vs : a.ks)[at] = z.scale;
}

// Claimed rows: `per` of them a block, KV8_FLY groups a thread in flight (us with 2 and 4, both launches: 20,011 rows x 8 x 128 bf16 36.1 and
// 37.3, 129 rows 6.5 and 8.8, 20,011 x 12 x 64 fp32 30.8 and 30.1).  fp32 groups pass at the rate of a copy (5.1 TB/s), bf16 ones, half the
// bytes, at 3.4: what a group costs besides its bytes (addresses, its scale, the rounding) counts there.
constexpr int KV8_FLY = 2, KV8_PER = 64;

template <typename T, int LPG>
__global__ void __launch_bounds__(256)
kv8_write_rows_kernel(Kv8Args a, int32_t per) {
    __shared__ int32_t s_place[KV8_PER];                    // -1: not written
    const int64_t row0 = block_of_lines() * per;
    if (row0 >= a.rows) return;
    const int rows = (int)min((int64_t)per, a.rows - row0), tid = threadIdx.x;
    const int l = tid % LPG, groups = rows * 2 * a.heads;   // (row, keys or values, head)
    const bool has = 8 * l < a.dim;
    constexpr int STEP = 256 / LPG;
    const float per_row = 1.f / (float)(2 * a.heads);       // (a block has fewer than 2^14 groups: the quotient below is exact)
    Raw8<T> x[KV8_FLY] = {};
    int32_t row[KV8_FLY], head[KV8_FLY];
    bool vals[KV8_FLY];
    auto fetch = [&](int g0) {                              // groups g0 + u STEP; behind the last one the last again
#pragma unroll
        for (int u = 0; u < KV8_FLY; ++u) {
            const int g = min(g0 + u * STEP, groups - 1);
            row[u] = (int)(((float)g + 0.5f) * per_row);
            const int h = g - row[u] * 2 * a.heads;
            vals[u] = h >= a.heads;
            head[u] = vals[u] ? h - a.heads : h;
            const int64_t r = row0 + row[u];
            if (has) load_raw((vals[u] ? (const T*)a.v + r * a.v_row + head[u] * a.v_head : (const T*)a.k + r * a.k_row + head[u] * a.k_head) + 8 * l, x[u]);
        }
    };
    fetch(tid / LPG);                                       // the rows come in beside the look at their places
    if (tid < rows) {
        const int64_t p = a.places_of[row0 + tid];
        s_place[tid] = p >= 0 && p < a.places && a.owner[p] == (int32_t)(row0 + tid) ? (int32_t)p : -1;
    }
    __syncthreads();
    if (tid < rows && s_place[tid] >= 0) a.owner[s_place[tid]] = -1;
    for (int g0 = tid / LPG; g0 < groups;) {
#pragma unroll
        for (int u = 0; u < KV8_FLY; ++u) {
            const uint32_t m = lanes_max<LPG>(largest8(0, x[u]));
            const int32_t place = s_place[row[u]];
            if (g0 + u * STEP >= groups || place < 0) continue;
            float f[8];
            values8(x[u], f);
            const Quant8 z(m);
            const int64_t at = (int64_t)place * a.heads + head[u];
            if (has) *reinterpret_cast<q8_u32x2*>((vals[u] ? a.v8 : a.k8) + at * a.dim + 8 * l) = pack8(z, f);
            if (l == 0) (vals[u] ? a.vs : a.ks)[at] = z.scale;
        }
        g0 += KV8_FLY * STEP;
        if (g0 < groups) fetch(g0);
    }
}

template <typename T, int LPG>
__global__ void __launch_bounds__(256)
kv8_read_kernel(Kv8Args a) {
    const int64_t g = (block_of_lines() * 256 + threadIdx.x) / LPG;
    const int l = threadIdx.x % LPG;
    const bool vals = blockIdx.z != 0;
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
        if constexpr (sizeof(T) == 2) {
            // The product has up to 31 bits.  Where fp32 puts it on the middle of two bf16 numbers (one in 2^16) its rest says which is the nearer one
            u16x2 low = {0xffff, 0xffff};                               // the low halves, the top bit turned over: 0 in the middle
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                low = __builtin_elementwise_min(low, __builtin_bit_cast(u16x2, __builtin_amdgcn_perm(__float_as_uint(x[i + 1]), __float_as_uint(x[i]), 0x05040100) ^ 0x80008000u));
            if (low[0] == 0 || low[1] == 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float rest = fmaf((float)(int8_t)(w[i / 4] >> (8 * (i % 4))), s, -x[i]);      // exact: all are multiples of 2^-149
                    const uint32_t u = __float_as_uint(x[i]), to = (rest > 0.f) == (x[i] > 0.f) ? u + 1 : u - 1;
                    if ((uint16_t)u == 0x8000 && fabsf(rest) > 0.f) x[i] = __uint_as_float(to);
                }
            }
        }
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
    if (a.rows <= KV8_LOOK) {
        kv8_write_kernel<T, LPG><<<dim3((unsigned)cdiv(a.rows * a.heads * LPG, 256), 2), 256, 0, st>>>(a);
        return check_launch("kv8_write_kernel");
    }
    kv8_claim_kernel<<<(unsigned)cdiv(a.rows, 256), 256, 0, st>>>(a);
    PS_TRY(check_launch("kv8_claim_kernel"));
    const int32_t per = std::max(1, std::min(KV8_PER, KV8_FLY * 256 / (2 * a.heads * LPG)));    // rows of a block: its groups in one go
    kv8_write_rows_kernel<T, LPG><<<block_lines(cdiv(a.rows, per)), 256, 0, st>>>(a, per);
    return check_launch("kv8_write_rows_kernel");
}
template <typename T, int LPG>
static int kv8_read_as(const Kv8Args& a, hipStream_t st) {
    kv8_read_kernel<T, LPG><<<block_lines(cdiv(a.rows * a.heads * LPG, 256), 2), 256, 0, st>>>(a);
    return check_launch("kv8_read_kernel");
}

}  // namespace pserve

static int check_device(const pserve_kv8_t* s, const char* who) {
    int dev;
    PS_CHECK_HIP(hipGetDevice(&dev));
    PS_REQUIRE(dev == s->device, "%s: the store is on device %d, the current one is %d", who, s->device, dev);
    return PSERVE_OK;
}

// What no launch is made for is refused before the first one, so that no claim is left behind: 2^28 groups
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
