// Linear layers in 8-bit integers (pserve_linear8_*), gfx950.
//
//   y[t][n] = (sum_k qx[t][k] qw[n][k]) * (sx[t] * sw[n]) + b[n] + residual[t][n]
//
// Two launches: the rows of x are quantised into the workspace (one pass over x, bound by memory), then the product runs on
// v_mfma_i32_32x32x32_i8, twice the rate of bf16.  Sums are exact in 32 bits: 127^2 * 131072 < 2^31.
// qw is kept as [N rounded up to 256][K rounded up to 128], qx as [rows][K rounded up to 128], both filled up with zeros, so a step
// of K is a row of 128 bytes in eight chunks, whatever K and N are; only the stores look at N.
#include "quant8.h"

using namespace pserve;

struct pserve_linear8_s {
    int32_t K = 0, N = 0, Kp = 0, Np = 0, dtype = 0;
    int device = 0;
    int8_t* w = nullptr;                        // [Np][Kp]
    float *scale = nullptr, *b = nullptr;       // [Np]
    pserve::DevicePool pool;
};

namespace pserve {

struct Linear8Args {
    const void *x, *res;
    void* y;
    int8_t* x8;                                 // [rows][Kp]
    float* x_scale;                             // [rows]
    const int8_t* w8;
    const float *w_scale, *b;
    int64_t rows, ldx;
    int32_t K, N, Kp, Np;
};

// ---- weights: largest magnitude of every column, then the transposed whole numbers
template <typename T>
__global__ void __launch_bounds__(256)
linear8_colmax_kernel(const T* w, int32_t K, int32_t N, uint32_t* amax) {
    const int n = blockIdx.x * 64 + (threadIdx.x & 63);
    uint32_t m = 0;
    if (n < N)
        for (int64_t k = blockIdx.y * 4 + (threadIdx.x >> 6); k < K; k += 4 * gridDim.y) m = max(m, abs_bits(load1(w + k * N + n)));
    if (n < N && m) atomicMax(amax + n, m);     // whole numbers: the order does not matter
}
template <typename T>
__global__ void __launch_bounds__(256)
linear8_pack_kernel(const T* w, int32_t K, int32_t N, int32_t Kp, const uint32_t* amax, int8_t* out, float* scale) {
    __shared__ int8_t tile[64][68];
    const int n0 = blockIdx.x * 64, k0 = blockIdx.y * 64, c = threadIdx.x & 63, r = threadIdx.x >> 6;
    const int n = n0 + c;
    const Quant8 z(n < N ? amax[n] : 0u);
    if (blockIdx.y == 0 && r == 0) scale[n] = z.scale;
    for (int i = r; i < 64; i += 4) tile[c][i] = n < N && k0 + i < K ? (int8_t)z(load1(w + (int64_t)(k0 + i) * N + n)) : (int8_t)0;
    __syncthreads();
    const int j = threadIdx.x >> 2, q = threadIdx.x & 3;
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint32_t*>(&tile[j][16 * q + 4 * i]);
    *reinterpret_cast<u32x4*>(out + (int64_t)(n0 + j) * Kp + k0 + 16 * q) = u32x4{v[0], v[1], v[2], v[3]};
}

// ---- rows of x: TPR threads a row, CH chunks of eight values a thread in registers; chunks behind those are read twice
template <typename T, int TPR, int CH, bool VEC>
__global__ void __launch_bounds__(256)
linear8_rows_kernel(Linear8Args a) {
    __shared__ uint32_t s_max[4];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (TPR < 256 && row >= a.rows) return;
    const T* x = (const T*)a.x + row * a.ldx;
    auto get = [&](int c, float (&v)[8]) {
        if (VEC) {
            if (8 * c < a.K) { load8(x + 8 * c, v); return; }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 8 * c + i < a.K ? load1(x + 8 * c + i) : 0.f;
        }
    };
    const int chunks = a.Kp / 8;
    float v[CH][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        get(t + i * TPR, v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, abs_bits(v[i][e]));
    }
    for (int c = t + CH * TPR; c < chunks; c += TPR) {
        float u[8];
        get(c, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, abs_bits(u[e]));
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
    if (TPR == 256) {
        if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
        __syncthreads();
        m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    }
    const Quant8 z(m);
    if (t == 0) a.x_scale[row] = z.scale;
    int8_t* o = a.x8 + row * a.Kp;
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (t + i * TPR < chunks) *reinterpret_cast<q8_u32x2*>(o + 8 * (t + i * TPR)) = pack8(z, v[i]);
    for (int c = t + CH * TPR; c < chunks; c += TPR) {
        float u[8];
        get(c, u);
        *reinterpret_cast<q8_u32x2*>(o + 8 * c) = pack8(z, u);
    }
}

template <typename T, bool VEC>
static int launch_rows_as(const Linear8Args& a, hipStream_t st) {
    if (a.Kp <= 1024) linear8_rows_kernel<T, 64, 2, VEC><<<(unsigned)cdiv(a.rows, 4), 256, 0, st>>>(a);
    else linear8_rows_kernel<T, 256, 4, VEC><<<(unsigned)a.rows, 256, 0, st>>>(a);
    return check_launch("linear8_rows_kernel");
}
template <typename T>
static int launch_rows(const Linear8Args& a, hipStream_t st) {
    const bool vec = a.K % 8 == 0 && a.ldx % (16 / sizeof(T)) == 0 && !((uintptr_t)a.x & 15);
    return vec ? launch_rows_as<T, true>(a, st) : launch_rows_as<T, false>(a, st);
}

// ---- the product: tiles of 128 rows x 128 channels, four wavefronts of 64 x 64, two stages of 128 values of K
__device__ __forceinline__ int l8_kperm(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }   // as in the bf16 layers

template <typename T>
__device__ __forceinline__ void l8_store(const Linear8Args& a, int64_t row, int n, const float (&v)[8], bool vec) {
    T* y = (T*)a.y + row * a.N + n;
    if (vec && n + 8 <= a.N) { store8(y, v); return; }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (n + i < a.N) store1(y + i, v[i]);
}

template <typename T>
__global__ void __launch_bounds__(256, 2)
linear8_tile_kernel(Linear8Args a, int m_tiles) {
    constexpr int BM = 128, BN = 128, LD = (BM + BN) / 32, STAGE_V = (BM + BN) * 8;
    __shared__ __attribute__((aligned(16))) uint8_t smem[2 * STAGE_V * 16];
    u32x4* ring = reinterpret_cast<u32x4*>(smem);           // [2][rows of x, rows of w][8 chunks], chunk ^ ((row >> 1) & 7)
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave & 1, wn = wave >> 1, fr = lane & 31, fh = lane >> 5;
    const int64_t m0 = (int64_t)(blockIdx.x % m_tiles) * BM;
    const int n0 = (int)(blockIdx.x / m_tiles) * BN;
    const int lc = lane & 7, lr = 8 * wave + (lane >> 3), gc = lc ^ ((lr >> 1) & 7);
    const int8_t* src[LD];
#pragma unroll
    for (int l = 0; l < LD; ++l) {
        const int r = lr + 32 * l;
        src[l] = (r < BM ? a.x8 + min(m0 + r, a.rows - 1) * a.Kp : a.w8 + (int64_t)(n0 + r - BM) * a.Kp) + gc * 16;
    }
    auto load_stage = [&](int kt, int stage) {
#pragma unroll
        for (int l = 0; l < LD; ++l)
            __builtin_amdgcn_global_load_lds((const void*)(src[l] + (int64_t)kt * 128), (lds_void*)(ring + stage * STAGE_V + (8 * wave + 32 * l) * 8), 16, 0, 0);
    };
    i32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    const int KT = a.Kp / 128;
    load_stage(0, 0);
    for (int kt = 0; kt < KT; ++kt) {
        if (kt + 1 < KT) {
            load_stage(kt + 1, (kt + 1) & 1);
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LD) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        }
        const u32x4* st = ring + (kt & 1) * STAGE_V;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            i32x4 fx[2], fw[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int rx = 64 * wm + 32 * i + fr, rw = 64 * wn + 32 * i + l8_kperm(fr);
                fx[i] = __builtin_bit_cast(i32x4, st[rx * 8 + ((2 * ks + fh) ^ ((rx >> 1) & 7))]);
                fw[i] = __builtin_bit_cast(i32x4, st[(BM + rw) * 8 + ((2 * ks + fh) ^ ((rw >> 1) & 7))]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[j], fx[i], acc[i][j], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");     // the stage is free for the next load
    }
    // the lane has row 32 i + fr and the channels 32 j + 16 c + 8 fh .. + 7
    const bool vec = a.N % (16 / sizeof(T)) == 0 && !((uintptr_t)a.y & 15);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t row = m0 + 64 * wm + 32 * i + fr;
        if (row >= a.rows) continue;
        const float sx = a.x_scale[row];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int n = n0 + 64 * wn + 32 * j + 16 * c + 8 * fh;
                if (n >= a.N) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] = (float)acc[i][j][8 * c + e] * (sx * a.w_scale[n + e]);
                    if (a.b) v[e] += a.b[n + e];
                    if (a.res && n + e < a.N) v[e] += load1((const T*)a.res + row * a.N + n + e);
                }
                l8_store<T>(a, row, n, v, vec);
            }
    }
}

template <typename T>
static int launch_tile(const Linear8Args& a, hipStream_t st) {
    const int64_t mt = cdiv(a.rows, 128), nt = cdiv(a.N, 128);
    linear8_tile_kernel<T><<<(unsigned)(mt * nt), 256, 0, st>>>(a, (int)mt);
    return check_launch("linear8_tile_kernel");
}

}  // namespace pserve

static size_t x8_bytes(const pserve_linear8_t* op, int64_t rows) { return (size_t)rows * op->Kp; }

extern "C" {

int pserve_linear8_create(int32_t K, int32_t N, int dtype, const void* w, const void* b, void* stream, pserve_linear8_t** out) {
    static const char who[] = "pserve_linear8_create";
    PS_REQUIRE(out, "%s: out is NULL", who);
    *out = nullptr;
    PS_REQUIRE(dtype == PSERVE_F32 || dtype == PSERVE_BF16, "%s: unknown dtype %d", who, dtype);
    PS_REQUIRE(K > 0 && N > 0 && K <= 131072 && N <= (1 << 24), "%s: %d x %d weights (K up to 131072)", who, K, N);
    PS_REQUIRE(w, "%s: NULL parameter", who);
    return guarded(who, [&]() -> int {
        std::unique_ptr<pserve_linear8_t> op(new pserve_linear8_t());
        op->K = K; op->N = N; op->dtype = dtype;
        op->Kp = (int32_t)cdiv(K, 128) * 128; op->Np = (int32_t)cdiv(N, 256) * 256;
        PS_CHECK_HIP(hipGetDevice(&op->device));
        hipStream_t st = (hipStream_t)stream;
        DevicePool tmp;
        uint32_t* amax = nullptr;
        PS_TRY(op->pool.alloc((void**)&op->w, (size_t)op->Np * op->Kp));
        PS_TRY(op->pool.alloc_t(&op->scale, op->Np));
        PS_TRY(tmp.alloc_t(&amax, op->Np));
        PS_CHECK_HIP(hipMemsetAsync(amax, 0, (size_t)op->Np * sizeof(uint32_t), st));
        const dim3 cg((unsigned)cdiv(N, 64), (unsigned)std::min<int64_t>(cdiv(K, 64), 64)), pg(op->Np / 64, op->Kp / 64);
        if (dtype == PSERVE_BF16) {
            linear8_colmax_kernel<<<cg, 256, 0, st>>>((const uint16_t*)w, K, N, amax);
            linear8_pack_kernel<<<pg, 256, 0, st>>>((const uint16_t*)w, K, N, op->Kp, amax, op->w, op->scale);
        } else {
            linear8_colmax_kernel<<<cg, 256, 0, st>>>((const float*)w, K, N, amax);
            linear8_pack_kernel<<<pg, 256, 0, st>>>((const float*)w, K, N, op->Kp, amax, op->w, op->scale);
        }
        PS_TRY(check_launch("linear8_pack_kernel"));
        if (b) {
            PS_TRY(op->pool.alloc_t(&op->b, op->Np));
            PS_CHECK_HIP(hipMemsetAsync(op->b, 0, (size_t)op->Np * sizeof(float), st));
            PS_TRY(pack_bias(b, op->b, N, dtype, st));
        }
        PS_CHECK_HIP(hipStreamSynchronize(st));
        *out = op.release();
        return PSERVE_OK;
    });
}

void pserve_linear8_free(pserve_linear8_t* op) { delete op; }

int pserve_linear8_workspace(const pserve_linear8_t* op, int64_t rows, size_t* bytes) {
    PS_REQUIRE(op && bytes, "pserve_linear8_workspace: NULL argument");
    PS_REQUIRE(rows >= 0 && rows <= INT32_MAX, "pserve_linear8_workspace: %lld rows", (long long)rows);
    *bytes = x8_bytes(op, rows) + (size_t)rows * sizeof(float);
    return PSERVE_OK;
}

int pserve_linear8_forward(const pserve_linear8_t* op, const void* x, int64_t ldx, int64_t rows, const void* residual,
                           void* workspace, size_t workspace_bytes, void* y, void* stream) {
    static const char who[] = "pserve_linear8_forward";
    PS_REQUIRE(op, "%s: NULL argument", who);
    size_t need = 0;
    PS_TRY(pserve_linear8_workspace(op, rows, &need));
    if (rows == 0) return PSERVE_OK;
    PS_REQUIRE(x && y && workspace, "%s: NULL buffer", who);
    PS_REQUIRE(ldx >= op->K, "%s: rows of x %lld apart, K = %d", who, (long long)ldx, op->K);
    PS_REQUIRE(workspace_bytes >= need && !((uintptr_t)workspace & 15), "%s: workspace of %zu bytes, %zu needed (16-byte aligned)", who, workspace_bytes, need);
    int dev;
    PS_CHECK_HIP(hipGetDevice(&dev));
    PS_REQUIRE(dev == op->device, "%s: the weights are on device %d, the current one is %d", who, op->device, dev);
    const uintptr_t es = dtype_size(op->dtype);
    PS_REQUIRE(!(((uintptr_t)x | (uintptr_t)y | (uintptr_t)residual) & (es - 1)), "%s: x, y or residual is not aligned to its type", who);
    PS_REQUIRE(cdiv(rows, 128) * cdiv(op->N, 128) <= INT32_MAX, "%s: too many tiles", who);
    Linear8Args a{};
    a.x = x; a.res = residual; a.y = y; a.rows = rows; a.ldx = ldx;
    a.x8 = (int8_t*)workspace; a.x_scale = (float*)((uint8_t*)workspace + x8_bytes(op, rows));
    a.w8 = op->w; a.w_scale = op->scale; a.b = op->b;
    a.K = op->K; a.N = op->N; a.Kp = op->Kp; a.Np = op->Np;
    hipStream_t st = (hipStream_t)stream;
    if (op->dtype == PSERVE_BF16) {
        PS_TRY(launch_rows<uint16_t>(a, st));
        return launch_tile<uint16_t>(a, st);
    }
    PS_TRY(launch_rows<float>(a, st));
    return launch_tile<float>(a, st);
}

}  // extern "C"
