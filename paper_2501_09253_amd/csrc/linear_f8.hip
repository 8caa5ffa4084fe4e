// Linear layers in 8-bit floating point with a scale for each block of 128 (pserve_linear_f8_*, pserve_f8_rows_*), gfx950.
//
//   y[t][n] = sum_b 2^(ex[t][b] + ew[n][b]) sum_{k in block b} vx[t][k] vw[n][k] + bias[n] + residual[t][n]
//
// Weights are kept as [N rounded up to 256][K rounded up to 128] numbers with their scale bytes, rows of x likewise, both filled up with
// zeros, so a step of K is one block: 128 bytes of a row and one scale, whatever K and N are; only the stores look at N.
// bf16 tensors: the scaled matrix instruction, which takes the powers of two beside the numbers.  Of eight neighbouring products it drops what lies
// below 2^-13 of the largest and adds what is left in fp32: 1e-4 of a result's size where the result's own rounding takes 1.7e-3.
// fp32 tensors: the numbers times their power of two are exact in bf16, and the bf16 instruction's sums are fp32 throughout.
#include "f8.h"

using namespace pserve;

struct pserve_linear_f8_s {
    int32_t K = 0, N = 0, Kp = 0, Np = 0, Sp = 0, dtype = 0;
    int device = 0;
    uint8_t *w = nullptr, *scale = nullptr;     // [Np][Kp], [Np][Sp]
    float* b = nullptr;                         // [Np]
    pserve::DevicePool pool;
};

namespace pserve {

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// 8 of a lane's 32 numbers times their scale, as bf16 (exact)
__device__ __forceinline__ bf16x8 f8_as_bf16(const i32x8& v, int q, int byte) {
    const float s = f8_scale_value((uint32_t)byte);
    bf16x8 o;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const bf16x2 lo = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)v[2 * q + h], s, false));
        const bf16x2 hi = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)v[2 * q + h], s, true));
        o[4 * h] = lo[0]; o[4 * h + 1] = lo[1]; o[4 * h + 2] = hi[0]; o[4 * h + 3] = hi[1];
    }
    return o;
}

struct LinearF8Args {
    const void *x, *res;
    void* y;
    uint8_t *x8, *sx;                           // [rows][Kp], [rows][Sp]
    const uint8_t *w8, *sw;
    const float* b;
    int64_t rows, ldx;
    int32_t K, N, Kp, Np, Sp;
};

// ---- weights: a tile of 128 of K x 64 channels, turned round in LDS
template <typename T>
__global__ void __launch_bounds__(256)
linear_f8_pack_kernel(const T* w, int32_t K, int32_t N, int32_t Kp, int32_t Sp, uint8_t* out, uint8_t* scale) {
    __shared__ float tile[64][132];
    __shared__ uint32_t s_max[4][64];
    const int n0 = blockIdx.x * 64, k0 = blockIdx.y * 128, c = threadIdx.x & 63, r = threadIdx.x >> 6, n = n0 + c;
    uint32_t m = 0;
    for (int i = r; i < 128; i += 4) {
        const float v = n < N && k0 + i < K ? load1(w + (int64_t)(k0 + i) * N + n) : 0.f;
        tile[c][i] = v;
        m = max(m, abs_bits(v));
    }
    s_max[r][c] = m;
    __syncthreads();
    const int j = threadIdx.x >> 2, q = threadIdx.x & 3;
    const F8Scale z(max(max(s_max[0][j], s_max[1][j]), max(s_max[2][j], s_max[3][j])));
    uint8_t* o = out + (int64_t)(n0 + j) * Kp + k0 + 32 * q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[j][32 * q + 8 * i + e];
        *reinterpret_cast<q8_u32x2*>(o + 8 * i) = z.pack8(v);
    }
    if (q == 0) scale[(int64_t)(n0 + j) * Sp + blockIdx.y] = (uint8_t)z.byte;
}

// ---- rows of x: a block of 128 is sixteen lanes of eight values each; blocks are numbered row by row
template <typename T, bool VEC>
__global__ void __launch_bounds__(256)
f8_rows_write_kernel(const T* x, int64_t ldx, int64_t rows, int32_t K, uint8_t* x8, uint8_t* sx) {
    const int Kp = f8_width(K), Sp = f8_scales(K), KB = Kp / 128, lane = threadIdx.x & 15;
    const int64_t blk = block_of_lines() * 16 + (threadIdx.x >> 4);
    if (blk >= rows * KB) return;               // (sixteen lanes in step)
    const int64_t row = blk / KB;
    const int b = (int)(blk - row * KB), c = 16 * b + lane;
    const T* p = x + row * ldx + 8 * c;
    float v[8];
    if (VEC) {
        if (8 * c < K) load8(p, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 8 * c + e < K ? load1(p + e) : 0.f;
    }
    const F8Scale z(lanes_max<16>(f8_largest(v)));
    *reinterpret_cast<q8_u32x2*>(x8 + row * Kp + 8 * c) = z.pack8(v);
    if (lane == 0) sx[row * Sp + b] = (uint8_t)z.byte;
    if (lane == 0 && b == 0)
        for (int i = KB; i < Sp; ++i) sx[row * Sp + i] = 127;
}

template <typename T>
__global__ void __launch_bounds__(256)
f8_rows_read_kernel(const uint8_t* x8, const uint8_t* sx, int64_t rows, int32_t K, T* x, int64_t ldx) {
    const int Kp = f8_width(K), Sp = f8_scales(K), words = (K + 3) / 4;
    const int64_t i = block_of_lines() * 256 + threadIdx.x, row = i / words;
    if (row >= rows) return;
    const int k = 4 * (int)(i - row * words);
    const float s = f8_scale_value(sx[row * Sp + k / 128]);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(x8 + row * Kp + k);
    const float v[4] = {__builtin_amdgcn_cvt_f32_fp8(w, 0), __builtin_amdgcn_cvt_f32_fp8(w, 1), __builtin_amdgcn_cvt_f32_fp8(w, 2), __builtin_amdgcn_cvt_f32_fp8(w, 3)};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (k + e < K) store1(x + row * ldx + k + e, v[e] * s);
}

template <typename T>
static int launch_rows_write(const void* x, int64_t ldx, int64_t rows, int32_t K, uint8_t* x8, uint8_t* sx, hipStream_t st) {
    const dim3 grid = block_lines(cdiv(rows * (f8_width(K) / 128), 16));
    if (K % 8 == 0 && ldx % (16 / sizeof(T)) == 0 && !((uintptr_t)x & 15)) f8_rows_write_kernel<T, true><<<grid, 256, 0, st>>>((const T*)x, ldx, rows, K, x8, sx);
    else f8_rows_write_kernel<T, false><<<grid, 256, 0, st>>>((const T*)x, ldx, rows, K, x8, sx);
    return check_launch("f8_rows_write_kernel");
}

// ---- the product: 16 MT rows x 16 NT channels, eight wavefronts that share K and read their operands from memory (a lane 32 bytes of a
// row's block), the next block's in flight; the sums meet in LDS, in a fixed order
template <typename T, int MT, int NT>
__global__ void __launch_bounds__(512)
linear_f8_few_kernel(LinearF8Args a, int m_tiles) {
    constexpr int BM = 16 * MT, BN = 16 * NT, RS = BN + 4, WV = 8;      // RS: values of a row in LDS
    __shared__ __attribute__((aligned(16))) float s_sum[WV][BM * RS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g4 = lane >> 4;
    const int64_t m0 = (int64_t)(blockIdx.x % m_tiles) * BM;
    const int n0 = (int)(blockIdx.x / m_tiles) * BN;
    const int KT = a.Kp / 128;                                          // blocks, dealt to the wavefronts in shares
    const int per = (KT + WV - 1) / WV, k0 = min(KT, wave * per), k1 = min(KT, k0 + per);
    const uint8_t *wp[NT], *xp[MT], *wsp[NT], *xsp[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t n = min(n0 + 16 * j + col, a.Np - 1);
        wp[j] = a.w8 + n * a.Kp + 32 * g4;
        wsp[j] = a.sw + n * a.Sp;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t r = min(m0 + 16 * i + col, a.rows - 1);
        xp[i] = a.x8 + r * a.Kp + 32 * g4;
        xsp[i] = a.sx + r * a.Sp;
    }
    f32x4 acc[MT][NT];
    i32x8 w[2][NT], x[2][MT];
    int ws[2][NT], xs[2][MT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto load = [&](int set, int k) {
        k = min(k, KT - 1);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            w[set][j] = *reinterpret_cast<const i32x8*>(wp[j] + (int64_t)k * 128);
            ws[set][j] = wsp[j][k];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            x[set][i] = *reinterpret_cast<const i32x8*>(xp[i] + (int64_t)k * 128);
            xs[set][i] = xsp[i][k];
        }
    };
    auto mma = [&](int set) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if constexpr (sizeof(T) == 2) {
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[set][j], x[set][i], acc[i][j], 0, 0, 0, ws[set][j], 0, xs[set][i]);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f8_as_bf16(w[set][j], q, ws[set][j]), f8_as_bf16(x[set][i], q, xs[set][i]), acc[i][j], 0, 0, 0);
                }
            }
    };
    if (k0 < k1) load(0, k0);
    for (int k = k0; k < k1; k += 2) {
        load(1, k + 1);
        mma(0);
        if (k + 1 >= k1) break;
        load(0, k + 2);
        mma(1);
    }
    // ---- the wavefronts' sums meet: the lane has row `col` of a tile and channels 4 g4 .. + 3
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(&s_sum[wave][(16 * i + col) * RS + 16 * j + 4 * g4]) = acc[i][j];
    __syncthreads();
    for (int idx = tid; idx < BM * BN / 4; idx += 64 * WV) {
        const int r = idx / (BN / 4), c = idx % (BN / 4) * 4, n = n0 + c;
        const int64_t row = m0 + r;
        if (row >= a.rows || n >= a.N) continue;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WV; ++i) s += *reinterpret_cast<const f32x4*>(&s_sum[i][r * RS + c]);
        const f32x4 b = a.b ? *reinterpret_cast<const f32x4*>(a.b + n) : f32x4{0.f, 0.f, 0.f, 0.f};
        T* yp = (T*)a.y + row * a.N + n;
        const T* rp = (const T*)a.res + row * a.N + n;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= a.N) break;
            float v = s[e] + b[e];
            if (a.res) v += load1(rp + e);
            store1(yp + e, v);
        }
    }
}

template <typename T, int MT, int NT>
static int launch_few(const LinearF8Args& a, hipStream_t st) {
    const int64_t mt = cdiv(a.rows, 16 * MT);
    linear_f8_few_kernel<T, MT, NT><<<(unsigned)(mt * cdiv(a.N, 16 * NT)), 512, 0, st>>>(a, (int)mt);
    return check_launch("linear_f8_few_kernel");
}

// ---- many tiles: WGM x WGN wavefronts of 32 TM rows x 32 TN channels, two stages of a block (128 of K) in LDS.
// A lane's operand of the 32 x 32 x 64 instruction is two 16-byte chunks of a row, chunk 4 ks + fh and 4 ks + 2 + fh of the block's eight (any
// order of K within a block does, the same for both operands).  The first operand's rows become the accumulators' rows, so the channels go
// first, in the order that leaves a lane with eight consecutive channels of one row of x.
__device__ __forceinline__ int lf_kperm(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

template <int WGM, int WGN, int TM, int TN>
struct LFCfg {
    static constexpr int NW = WGM * WGN, WM = 32 * TM, WN = 32 * TN, BM = WGM * WM, BN = WGN * WN;
    static constexpr int STAGE = (BM + BN) * 128;           // bytes
    static constexpr int LDS = 2 * STAGE + 2 * 4 * (BM + BN);       // two stages; scales of four blocks, of this group and the next
    static_assert(64 * NW == BM + BN, "a thread loads the scales of a row");
    static_assert(STAGE >= NW * 4096, "the output staging (4 KB a wavefront) reuses a stage");
};

template <typename T, bool RES, bool VEC, int WGM, int WGN, int TM, int TN>
__global__ void __launch_bounds__(64 * WGM * WGN, 2)
linear_f8_tile_kernel(LinearF8Args a, int m_tiles, int total) {
    using Cfg = LFCfg<WGM, WGN, TM, TN>;
    constexpr int NW = Cfg::NW, WM = Cfg::WM, WN = Cfg::WN, BM = Cfg::BM, BN = Cfg::BN;
    constexpr int RP = 8 * NW, A_LD = BM / RP, B_LD = BN / RP, LD = A_LD + B_LD, STAGE_V = Cfg::STAGE / 16;
    constexpr int GM = 8;                                   // row tiles of a group, see below
    extern __shared__ __attribute__((aligned(16))) uint8_t lf_smem[];
    u32x4* ring = reinterpret_cast<u32x4*>(lf_smem);        // [2][rows of x, rows of w][8 chunks], chunk ^ ((row >> 1) & 7)
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WGM, wn = wave / WGM, fr = lane & 31, fh = lane >> 5;
    const int n_tiles = total / m_tiles, KT = a.Kp / 128;

    // Tiles are numbered in groups of GM row tiles, rows fastest; XCD x (block id mod 8) takes the x-th eighth of the numbers, so
    // the blocks of an XCD run on neighbouring tiles and share the panels in its L2.
    const int xcd = blockIdx.x & 7, t_end = (int)((int64_t)total * (xcd + 1) / 8), t_step = gridDim.x >> 3;
    int t = (int)((int64_t)total * xcd / 8) + (blockIdx.x >> 3);
    if (t >= t_end) return;

    const int lc = lane & 7, lr = 8 * wave + (lane >> 3), gc = lc ^ ((lr >> 1) & 7);
    int a_off[A_LD], b_off[B_LD];                           // byte offsets from the tile's first row
    const uint8_t *a_base, *b_base;
    const uint8_t* s_base;                                  // scales of the thread's row
    int64_t m0 = 0;
    int n0 = 0;
    auto decode = [&](int tt) {
        const int grp = tt / (GM * n_tiles), r = tt - grp * (GM * n_tiles), gm = min(GM, m_tiles - grp * GM), nt = r / gm;
        m0 = (int64_t)(grp * GM + r - nt * gm) * BM;
        n0 = nt * BN;
    };
    const int rowA = wm * WM + fr, rowB = wn * WN + lf_kperm(fr);
    auto setup = [&]() {
        a_base = a.x8 + m0 * a.Kp;
        b_base = a.w8 + (int64_t)n0 * a.Kp;
        const int last = (int)min((int64_t)BM, a.rows - m0) - 1, lastB = a.Np - 1 - n0;
#pragma unroll
        for (int l = 0; l < A_LD; ++l) a_off[l] = min(lr + l * RP, last) * a.Kp + gc * 16;
#pragma unroll
        for (int l = 0; l < B_LD; ++l) b_off[l] = min(lr + l * RP, lastB) * a.Kp + gc * 16;
        s_base = tid < BM ? a.sx + (m0 + min(tid, last)) * a.Sp : a.sw + (int64_t)(n0 + min(tid - BM, lastB)) * a.Sp;
    };
    uint32_t* s_scale = reinterpret_cast<uint32_t*>(lf_smem + 2 * Cfg::STAGE);      // [2][rows of x, rows of w] words of four blocks
    auto load_scales = [&](int group) {
        __builtin_amdgcn_global_load_lds((const void*)(s_base + 4 * group), (lds_void*)(s_scale + (group & 1) * (BM + BN) + wave * 64), 4, 0, 0);
    };
    auto load_stage = [&](int kt, int stage) {
        u32x4* dst = ring + stage * STAGE_V + wave * 64;
        const uint8_t *ap = a_base + (int64_t)kt * 128, *bp = b_base + (int64_t)kt * 128;
#pragma unroll
        for (int l = 0; l < A_LD; ++l) __builtin_amdgcn_global_load_lds((const void*)(ap + a_off[l]), (lds_void*)(dst + l * (64 * NW)), 16, 0, 0);
#pragma unroll
        for (int l = 0; l < B_LD; ++l) __builtin_amdgcn_global_load_lds((const void*)(bp + b_off[l]), (lds_void*)(dst + BM * 8 + l * (64 * NW)), 16, 0, 0);
    };
    const u32x4 *pA = ring + rowA * 8, *pB = ring + BM * 8 + rowB * 8;
    const int swA = (rowA >> 1) & 7, swB = (rowB >> 1) & 7;
    // One load instruction a call, so that the refill of a stage is spread over the matrix instructions behind the barrier that frees it
    auto load_one = [&](int kt, int stage, int l) {
        u32x4* dst = ring + stage * STAGE_V + wave * 64;
        if (l < A_LD) __builtin_amdgcn_global_load_lds((const void*)(a_base + (int64_t)kt * 128 + a_off[l < A_LD ? l : 0]), (lds_void*)(dst + l * (64 * NW)), 16, 0, 0);
        else __builtin_amdgcn_global_load_lds((const void*)(b_base + (int64_t)kt * 128 + b_off[l >= A_LD ? l - A_LD : 0]),
                                              (lds_void*)(dst + BM * 8 + (l - A_LD) * (64 * NW)), 16, 0, 0);
    };
    i32x8 fa[2][TM], fb[TN];
    auto fragment = [&](const u32x4* row, int ks, int sw) {
        const u32x4 lo = row[(4 * ks + fh) ^ sw], hi = row[(4 * ks + 2 + fh) ^ sw];
        return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    auto read_a = [&](int stage, int ks, int i) { fa[ks][i] = fragment(pA + stage * STAGE_V + i * 256, ks, swA); };
    auto read_b = [&](int stage, int ks, int j) { fb[j] = fragment(pB + stage * STAGE_V + j * 256, ks, swB); };
    int xa[TM], xb[TN], xa_next[TM], xb_next[TN];           // scale bytes of four blocks, and of the next four
    auto mma = [&](int ks, int i, int j, f32x16& c) {
        if constexpr (sizeof(T) == 2) {
            c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j], fa[ks][i], c, 0, 0, 0, xb[j], 0, xa[i]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f8_as_bf16(fb[j], q, xb[j] & 255), f8_as_bf16(fa[ks][i], q, xa[i] & 255), c, 0, 0, 0);
        }
        asm volatile("" : "+v"(c));                         // (it stays here: else the compiler sinks it past the branches around the loads)
    };
    constexpr int NM = TM * TN;                             // matrix instructions of half a block
    constexpr int LPS = (LD + 2 * NM - TM - 1) / (2 * NM - TM);     // loads behind one of them

    auto read_scales = [&](int group, int (&pa)[TM], int (&pb)[TN]) {
        const uint32_t* p = s_scale + (group & 1) * (BM + BN);
#pragma unroll
        for (int i = 0; i < TM; ++i) pa[i] = (int)p[rowA + 32 * i];
#pragma unroll
        for (int j = 0; j < TN; ++j) pb[j] = (int)p[BM + rowB + 32 * j];
    };

    decode(t);
    setup();
    load_stage(0, 0);
    load_scales(0);
    if (KT > 1) load_stage(1, 1);
#pragma unroll 1
    for (;;) {
        f32x16 acc[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");           // the first two blocks have landed
#pragma unroll
        for (int i = 0; i < TM; ++i) read_a(0, 0, i);
#pragma unroll
        for (int j = 0; j < TN; ++j) read_b(0, 0, j);
        read_scales(0, xa, xb);
#pragma unroll 1
        for (int kt = 0; kt < KT; ++kt) {
            const int cur = kt & 1, nxt = cur ^ 1;
            const bool refill = kt + 2 < KT, late = kt > 0 && kt + 1 < KT;
            const bool turn = (kt & 3) == 3;
            if ((kt & 3) == 0 && kt + 4 < KT) load_scales(kt / 4 + 1);
            if (turn) read_scales(kt / 4 + 1, xa_next, xb_next);        // (where there is a next group, in three steps' time it has landed)
            // first half: the second half's operands come in, a channel tile's as soon as its last instruction is out
#pragma unroll
            for (int q = 0; q < NM; ++q) {
                const int j = q / TM, i = q % TM, sl = NM - TM + q;
                mma(0, i, j, acc[i][j]);
                if (q < TM) read_a(cur, 1, q);
                if (i == TM - 1) read_b(cur, 1, j);
                if (late) {
#pragma unroll
                    for (int l = 0; l < LD; ++l) if (l / LPS == sl) load_one(kt + 1, nxt, l);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            // second half: behind its first instructions every operand of the stage has been read and the next stage has landed (what is read
            // behind the last step is not used)
#pragma unroll
            for (int q = 0; q < NM; ++q) {
                const int j = q / TM, i = q % TM;
                mma(1, i, j, acc[i][j]);
                if (q == TM - 1) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
                if (q >= TM - 1) {
                    if (q < 2 * TM - 1) read_a(nxt, 0, q - (TM - 1));
                    if (i == TM - 1) read_b(nxt, 0, j);
                    if (refill && q >= TM) {
#pragma unroll
                        for (int l = 0; l < LD; ++l) if (l / LPS == q - TM) load_one(kt + 2, cur, l);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) xa[i] = turn ? xa_next[i] : (int)((uint32_t)xa[i] >> 8);
#pragma unroll
            for (int j = 0; j < TN; ++j) xb[j] = turn ? xb_next[j] : (int)((uint32_t)xb[j] >> 8);
        }
        // ---- output in pieces of 32 rows x 128 bytes, through the second stage
        const int64_t r0 = m0 + wm * WM;
        const int c0 = n0 + wn * WN;
        constexpr int CV = 16 / sizeof(T), PC = 8 * CV;     // values of a 16-byte chunk, columns of a piece
        constexpr int PJ = PC / 32, NP = TN / PJ;           // accumulator tiles of a piece, pieces of 32 rows
        const int nt = t + t_step;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // every wavefront has read its last fragments
        if (nt < t_end) {                                   // the first step of the next tile comes in beside the end of this one
            decode(nt);
            setup();
            load_stage(0, 0);
            load_scales(0);
        }
        u32x4* ep = ring + STAGE_V + wave * 256;            // [32 rows][8 chunks], chunk ^ ((row >> 1) & 7)
        const int er = lane >> 3, ec = lane & 7, sw = (fr >> 1) & 7;
        // chunk of the lane's 16-byte word q of a piece: words 2 jj + c (bf16), 2 c + h (fp32)
        auto chunk = [&](int q) { return (sizeof(T) == 2 ? 2 * q + fh : 4 * (q >> 1) + 2 * fh + (q & 1)) ^ sw; };
        // value `lane % PC` of row r of a piece
        constexpr int RI = 64 / PC;                         // rows an instruction covers where the rows are off the 16-byte grid
        auto cell = [&](int r) -> T* { return reinterpret_cast<T*>(ep + r * 8 + (((lane % PC) / CV) ^ ((r >> 1) & 7))) + lane % CV; };
#pragma unroll
        for (int p = 0; p < TM * NP; ++p) {
            const int i = p / NP, jp = p % NP, pcol = c0 + PC * jp;
            if (pcol >= a.N) continue;
            const bool in = pcol + lane % PC < a.N;
            u32x4 rres[4];
            if constexpr (RES) {                            // the residual as the accumulators lie, through the staging
                if constexpr (VEC) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int rr = 8 * k + er, n = pcol + CV * ec;
                        const int64_t row = min(r0 + 32 * i + rr, a.rows - 1);
                        ep[rr * 8 + (ec ^ ((rr >> 1) & 7))] = *reinterpret_cast<const u32x4*>((const T*)a.res + row * a.N + (n < a.N ? n : 0));
                    }
                } else {
#pragma unroll 8
                    for (int r = lane / PC; r < 32; r += RI) {
                        const int64_t row = r0 + 32 * i + r;
                        *cell(r) = in && row < a.rows ? ((const T*)a.res)[row * a.N + pcol + lane % PC] : T(0);
                    }
                }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int q = 0; q < 4; ++q) rres[q] = ep[fr * 8 + chunk(q)];
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll
            for (int jj = 0; jj < PJ; ++jj)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int n = pcol + 32 * jj + 16 * c + 8 * fh;
                    float v[8], b[8];
                    if (a.b && n < a.Np) load8(a.b + n, b);
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e) b[e] = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[e] = acc[i][jp * PJ + jj][8 * c + e] + b[e];
                        if constexpr (RES && sizeof(T) == 2) {
                            const uint32_t r = rres[2 * jj + c][e / 2];
                            v[e] += e & 1 ? __uint_as_float(r & 0xffff0000u) : __uint_as_float(r << 16);
                        } else if constexpr (RES) {
                            v[e] += __uint_as_float(rres[2 * c + e / 4][e % 4]);
                        }
                    }
                    if constexpr (sizeof(T) == 2) {
                        ep[fr * 8 + chunk(2 * jj + c)] = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            ep[fr * 8 + chunk(2 * c + h)] = u32x4{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
                    }
                }
            __builtin_amdgcn_wave_barrier();
            if constexpr (VEC) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int rr = 8 * k + er, n = pcol + CV * ec;
                    const int64_t row = r0 + 32 * i + rr;
                    const u32x4 o = ep[rr * 8 + (ec ^ ((rr >> 1) & 7))];
                    // (past the L2, which holds the panels)
                    if (row < a.rows && n < a.N) __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>((T*)a.y + row * a.N + n));
                }
            } else {
#pragma unroll 8
                for (int r = lane / PC; r < 32; r += RI) {
                    const int64_t row = r0 + 32 * i + r;
                    if (in && row < a.rows) ((T*)a.y)[row * a.N + pcol + lane % PC] = *cell(r);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (nt >= t_end) break;
        t = nt;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // the staging is done with
        if (KT > 1) load_stage(1, 1);
    }
}

template <typename T, bool RES, bool VEC, int WGM, int WGN, int TM, int TN>
static int launch_tile_as(const LinearF8Args& a, hipStream_t st) {
    using Cfg = LFCfg<WGM, WGN, TM, TN>;
    PS_SET_LDS_ONCE((linear_f8_tile_kernel<T, RES, VEC, WGM, WGN, TM, TN>), Cfg::LDS);
    const int64_t mt = cdiv(a.rows, Cfg::BM), total = mt * cdiv(a.N, Cfg::BN);
    const unsigned grid = (unsigned)(8 * cdiv(std::min<int64_t>(total, Cfg::LDS > 80 * 1024 ? 256 : 512), 8));
    linear_f8_tile_kernel<T, RES, VEC, WGM, WGN, TM, TN><<<grid, 64 * Cfg::NW, Cfg::LDS, st>>>(a, (int)mt, (int)total);
    return check_launch("linear_f8_tile_kernel");
}
template <typename T, bool RES, bool VEC>
static int launch_tile_vec(const LinearF8Args& a, hipStream_t st) {
    if (cdiv(a.rows, 256) * cdiv(a.N, 256) >= 256) return launch_tile_as<T, RES, VEC, 4, 2, 2, 4>(a, st);
    return launch_tile_as<T, RES, VEC, 2, 2, 2, 2>(a, st);
}
template <typename T>
static int launch_tile(const LinearF8Args& a, hipStream_t st) {
    const bool vec = a.N % (16 / sizeof(T)) == 0 && !(((uintptr_t)a.y | (uintptr_t)a.res) & 15);
    if (a.res) return vec ? launch_tile_vec<T, true, true>(a, st) : launch_tile_vec<T, true, false>(a, st);
    return vec ? launch_tile_vec<T, false, true>(a, st) : launch_tile_vec<T, false, false>(a, st);
}

template <typename T>
static int product(const LinearF8Args& a, hipStream_t st) {
    if (a.rows <= 32) return launch_few<T, 1, 1>(a, st);
    if (cdiv(a.rows, 128) * cdiv(a.N, 128) <= 64) return launch_few<T, 2, 2>(a, st);
    return launch_tile<T>(a, st);
}

static int rows_ok(const char* who, int64_t rows, int32_t K) {
    PS_REQUIRE(rows >= 0 && rows < (1 << 26), "%s: %lld rows (fewer than 2^26)", who, (long long)rows);
    PS_REQUIRE(K > 0 && K <= 131072, "%s: K = %d (1 .. 131072)", who, K);
    return PSERVE_OK;
}

static int run_product(const char* who, const pserve_linear_f8_t* op, LinearF8Args& a, const void* rows8, const void* residual, void* y, hipStream_t st) {
    PS_REQUIRE(cdiv(a.rows, 32) * cdiv(op->N, 32) <= INT32_MAX, "%s: too many tiles", who);
    int dev;
    PS_CHECK_HIP(hipGetDevice(&dev));
    PS_REQUIRE(dev == op->device, "%s: the weights are on device %d, the current one is %d", who, op->device, dev);
    const uintptr_t es = dtype_size(op->dtype);
    PS_REQUIRE(!(((uintptr_t)a.x | (uintptr_t)y | (uintptr_t)residual) & (es - 1)), "%s: x, y or residual is not aligned to its type", who);
    a.x8 = (uint8_t*)rows8; a.sx = a.x8 + (size_t)a.rows * op->Kp;
    a.res = residual; a.y = y;
    a.w8 = op->w; a.sw = op->scale; a.b = op->b;
    a.K = op->K; a.N = op->N; a.Kp = op->Kp; a.Np = op->Np; a.Sp = op->Sp;
    if (a.x) {
        if (op->dtype == PSERVE_BF16) PS_TRY(launch_rows_write<uint16_t>(a.x, a.ldx, a.rows, a.K, a.x8, a.sx, st));
        else PS_TRY(launch_rows_write<float>(a.x, a.ldx, a.rows, a.K, a.x8, a.sx, st));
    }
    return op->dtype == PSERVE_BF16 ? product<uint16_t>(a, st) : product<float>(a, st);
}

}  // namespace pserve

extern "C" {

int pserve_f8_rows_bytes(int64_t rows, int32_t K, size_t* bytes) {
    PS_REQUIRE(bytes, "pserve_f8_rows_bytes: NULL argument");
    PS_TRY(rows_ok("pserve_f8_rows_bytes", rows, K));
    *bytes = f8_bytes(rows, K);
    return PSERVE_OK;
}

int pserve_f8_rows_write(const void* x, int64_t ldx, int64_t rows, int32_t K, int dtype, void* rows8, void* stream) {
    static const char who[] = "pserve_f8_rows_write";
    PS_TRY(rows_ok(who, rows, K));
    PS_REQUIRE(dtype == PSERVE_F32 || dtype == PSERVE_BF16, "%s: unknown dtype %d", who, dtype);
    if (rows == 0) return PSERVE_OK;
    PS_REQUIRE(x && rows8, "%s: NULL buffer", who);
    PS_REQUIRE(ldx >= K || rows == 1, "%s: rows of x %lld apart, K = %d", who, (long long)ldx, K);
    PS_REQUIRE(!((uintptr_t)rows8 & 15) && !((uintptr_t)x & (dtype_size(dtype) - 1)), "%s: rows8 is not 16-byte aligned, or x not to its type", who);
    uint8_t *v = (uint8_t*)rows8, *s = v + (size_t)rows * f8_width(K);
    hipStream_t st = (hipStream_t)stream;
    return dtype == PSERVE_BF16 ? launch_rows_write<uint16_t>(x, ldx, rows, K, v, s, st) : launch_rows_write<float>(x, ldx, rows, K, v, s, st);
}

int pserve_f8_rows_read(const void* rows8, int64_t rows, int32_t K, int dtype, void* x, int64_t ldx, void* stream) {
    static const char who[] = "pserve_f8_rows_read";
    PS_TRY(rows_ok(who, rows, K));
    PS_REQUIRE(dtype == PSERVE_F32 || dtype == PSERVE_BF16, "%s: unknown dtype %d", who, dtype);
    if (rows == 0) return PSERVE_OK;
    PS_REQUIRE(x && rows8, "%s: NULL buffer", who);
    PS_REQUIRE(ldx >= K || rows == 1, "%s: rows of x %lld apart, K = %d", who, (long long)ldx, K);
    PS_REQUIRE(!((uintptr_t)rows8 & 15) && !((uintptr_t)x & (dtype_size(dtype) - 1)), "%s: rows8 is not 16-byte aligned, or x not to its type", who);
    const uint8_t *v = (const uint8_t*)rows8, *s = v + (size_t)rows * f8_width(K);
    const dim3 grid = block_lines(cdiv(rows * cdiv(K, 4), 256));
    hipStream_t st = (hipStream_t)stream;
    if (dtype == PSERVE_BF16) f8_rows_read_kernel<<<grid, 256, 0, st>>>(v, s, rows, K, (uint16_t*)x, ldx);
    else f8_rows_read_kernel<<<grid, 256, 0, st>>>(v, s, rows, K, (float*)x, ldx);
    return check_launch("f8_rows_read_kernel");
}

int pserve_linear_f8_create(int32_t K, int32_t N, int dtype, const void* w, const void* b, void* stream, pserve_linear_f8_t** out) {
    static const char who[] = "pserve_linear_f8_create";
    PS_REQUIRE(out, "%s: out is NULL", who);
    *out = nullptr;
    PS_REQUIRE(dtype == PSERVE_F32 || dtype == PSERVE_BF16, "%s: unknown dtype %d", who, dtype);
    PS_REQUIRE(K > 0 && N > 0 && K <= 131072 && N <= (1 << 24), "%s: %d x %d weights (K up to 131072, N up to 2^24)", who, K, N);
    PS_REQUIRE(w, "%s: NULL parameter", who);
    PS_REQUIRE(!(((uintptr_t)w | (uintptr_t)b) & (dtype_size(dtype) - 1)), "%s: w or b is not aligned to its type", who);
    return guarded(who, [&]() -> int {
        std::unique_ptr<pserve_linear_f8_t> op(new pserve_linear_f8_t());
        op->K = K; op->N = N; op->dtype = dtype;
        op->Kp = f8_width(K); op->Np = (int32_t)cdiv(N, 256) * 256; op->Sp = f8_scales(K);
        PS_CHECK_HIP(hipGetDevice(&op->device));
        hipStream_t st = (hipStream_t)stream;
        PS_TRY(op->pool.alloc((void**)&op->w, (size_t)op->Np * op->Kp));
        PS_TRY(op->pool.alloc((void**)&op->scale, (size_t)op->Np * op->Sp));
        PS_CHECK_HIP(hipMemsetAsync(op->scale, 127, (size_t)op->Np * op->Sp, st));
        const dim3 grid(op->Np / 64, op->Kp / 128);
        if (dtype == PSERVE_BF16) linear_f8_pack_kernel<<<grid, 256, 0, st>>>((const uint16_t*)w, K, N, op->Kp, op->Sp, op->w, op->scale);
        else linear_f8_pack_kernel<<<grid, 256, 0, st>>>((const float*)w, K, N, op->Kp, op->Sp, op->w, op->scale);
        PS_TRY(check_launch("linear_f8_pack_kernel"));
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

void pserve_linear_f8_free(pserve_linear_f8_t* op) { delete op; }

int pserve_linear_f8_workspace(const pserve_linear_f8_t* op, int64_t rows, size_t* bytes) {
    PS_REQUIRE(op && bytes, "pserve_linear_f8_workspace: NULL argument");
    PS_TRY(rows_ok("pserve_linear_f8", rows, op->K));
    *bytes = f8_bytes(rows, op->K);
    return PSERVE_OK;
}

int pserve_linear_f8_forward(const pserve_linear_f8_t* op, const void* x, int64_t ldx, int64_t rows, const void* residual, void* workspace,
                             size_t workspace_bytes, void* y, void* stream) {
    static const char who[] = "pserve_linear_f8_forward";
    PS_REQUIRE(op, "%s: NULL argument", who);
    size_t need = 0;
    PS_TRY(pserve_linear_f8_workspace(op, rows, &need));
    if (rows == 0) return PSERVE_OK;
    PS_REQUIRE(x && y && workspace, "%s: NULL buffer", who);
    PS_REQUIRE(ldx >= op->K || rows == 1, "%s: rows of x %lld apart, K = %d", who, (long long)ldx, op->K);
    PS_REQUIRE(workspace_bytes >= need && !((uintptr_t)workspace & 15), "%s: workspace of %zu bytes, %zu needed (16-byte aligned)", who, workspace_bytes, need);
    LinearF8Args a{};
    a.x = x; a.rows = rows; a.ldx = ldx;
    return run_product(who, op, a, workspace, residual, y, (hipStream_t)stream);
}

int pserve_linear_f8_forward_rows(const pserve_linear_f8_t* op, const void* rows8, int64_t rows, const void* residual, void* y, void* stream) {
    static const char who[] = "pserve_linear_f8_forward_rows";
    PS_REQUIRE(op, "%s: NULL argument", who);
    PS_TRY(rows_ok(who, rows, op->K));
    if (rows == 0) return PSERVE_OK;
    PS_REQUIRE(rows8 && y, "%s: NULL buffer", who);
    PS_REQUIRE(!((uintptr_t)rows8 & 15), "%s: rows8 is not 16-byte aligned", who);
    LinearF8Args a{};
    a.rows = rows;
    return run_product(who, op, a, rows8, residual, y, (hipStream_t)stream);
}

}  // extern "C"
