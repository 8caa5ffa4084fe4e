// Linear layers in 8-bit floating point with a scale for each block of 128 (pserve_linear_f8_*, pserve_f8_rows_*), gfx950.
//
//   y[t][n] = sum_b 2^(ex[t][b] + ew[n][b]) sum_{k in block b} vx[t][k] vw[n][k] + bias[n] + residual[t][n]
//
// Weights are kept as [N rounded up to 256][K rounded up to 128] numbers with their scale bytes, rows of x likewise, both filled up with
// zeros, so a step of K is one block: 128 bytes of a row and one scale, whatever K and N are; only the stores look at N.
// bf16 tensors: the scaled matrix instruction, which takes the powers of two beside the numbers.  Of eight neighbouring products it drops what lies
// below 2^-13 of the largest and adds what is left in fp32.  Of normal values (12 x 4096 x 4096 .. 12,544 x 1536 x 6144) the sums are 1.5e-5 .. 1.9e-5 of a result's size
// off, 4e-6 where all products have one sign; the result's own rounding takes 1.7e-3, and comes out one step apart for one result in a hundred, which makes
// 2e-4 .. 3e-4 between rounded results of these and of fp32 sums.
// fp32 tensors: the numbers times their power of two are exact in bf16, and the bf16 instruction's sums are fp32 throughout.
// Few rows are bound by how fast a CU takes in operands, few tiles by the way of a tile's first operands and its outputs, many by the matrix
// cores (8192^3 427 us, 2,570 TFLOP/s, the clock at 1.7 GHz under their load) and, where K is short, by the outputs and residuals that a tile
// moves while they wait (12,544 x 1536 x 6144 with a residual 142 us beside its rows' rounding, 1,670 TFLOP/s, and 147 .. 181 product
// behind product, by the clock: they are busy 44 % of the time).
#include "f8.h"

using namespace pserve;

struct pserve_linear_f8_s {
    int32_t K = 0, N = 0, Kp = 0, Np = 0, dtype = 0;
    int device = 0;
    uint8_t *w = nullptr, *scale = nullptr;     // [Np][Kp], [words of four blocks][Np][4]
    float* b = nullptr;                         // [Np]
    pserve::DevicePool pool;
};

namespace pserve {

typedef __attribute__((ext_vector_type(8))) int i32x8;

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
    uint8_t *x8, *sx;                           // [rows][Kp], [words of four blocks][rows][4]
    const uint8_t *w8, *sw;
    const float* b;
    int64_t rows, ldx;
    int32_t K, N, Kp, Np;
};

// ---- weights: a tile of 128 of K x 64 channels, turned round in LDS
template <typename T>
__global__ void __launch_bounds__(256)
linear_f8_pack_kernel(const T* w, int32_t K, int32_t N, int32_t Kp, int32_t Np, uint8_t* out, uint8_t* scale) {
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
        z.pack(v, o + 8 * i);
    }
    if (q == 0) scale[f8_scale_at(Np, n0 + j, blockIdx.y)] = (uint8_t)z.byte;
}

// ---- rows of x: a block of 128 is sixteen lanes of eight values each; blocks are numbered row by row
template <typename T, bool EVEN>
__global__ void __launch_bounds__(256)
f8_rows_write_kernel(const T* x, int64_t ldx, int64_t rows, int32_t K, uint8_t* x8, uint8_t* sx) {
    const int Kp = f8_width(K), Sp = f8_scales(K), KB = Kp / 128, lane = threadIdx.x & 15;
    const int64_t blk = block_of_lines() * 16 + (threadIdx.x >> 4);
    if (blk >= rows * KB) return;               // (sixteen lanes in step)
    const int64_t row = blk / KB;
    const int b = (int)(blk - row * KB), c = 16 * b + lane;
    const T* p = x + row * ldx + 8 * c;
    typedef typename AnyPiece<T>::type Any;
    Raw8<T> r;
    if (EVEN ? 8 * c < K : 8 * c + 8 <= K) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) r.w[h] = *reinterpret_cast<const Any*>(p + h * (16 / sizeof(T)));
    } else {
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = !EVEN && 8 * c + e < K ? p[e] : T(0);
        __builtin_memcpy(&r, v, sizeof r);
    }
    const F8Scale z(lanes_max<16>(largest8(0u, r)));
    *reinterpret_cast<q8_u32x2*>(x8 + row * Kp + 8 * c) = z.pack8(r);
    if (lane == 0) sx[f8_scale_at(rows, row, b)] = (uint8_t)z.byte;
    if (lane == 0 && b == 0)
        for (int i = KB; i < Sp; ++i) sx[f8_scale_at(rows, row, i)] = 127;
}

template <typename T>
__global__ void __launch_bounds__(256)
f8_rows_read_kernel(const uint8_t* x8, const uint8_t* sx, int64_t rows, int32_t K, T* x, int64_t ldx) {
    const int Kp = f8_width(K), words = (K + 3) / 4;
    const int64_t i = block_of_lines() * 256 + threadIdx.x, row = i / words;
    if (row >= rows) return;
    const int k = 4 * (int)(i - row * words);
    const float s = f8_scale_value(sx[f8_scale_at(rows, row, k / 128)]);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(x8 + row * Kp + k);
    const float v[4] = {__builtin_amdgcn_cvt_f32_fp8(w, 0), __builtin_amdgcn_cvt_f32_fp8(w, 1), __builtin_amdgcn_cvt_f32_fp8(w, 2), __builtin_amdgcn_cvt_f32_fp8(w, 3)};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (k + e < K) store1(x + row * ldx + k + e, v[e] * s);
}

template <typename T>
static int launch_rows_write(const void* x, int64_t ldx, int64_t rows, int32_t K, uint8_t* x8, uint8_t* sx, hipStream_t st) {
    const dim3 grid = block_lines(cdiv(rows * (f8_width(K) / 128), 16));
    if (K % 8 == 0) f8_rows_write_kernel<T, true><<<grid, 256, 0, st>>>((const T*)x, ldx, rows, K, x8, sx);
    else f8_rows_write_kernel<T, false><<<grid, 256, 0, st>>>((const T*)x, ldx, rows, K, x8, sx);
    return check_launch("f8_rows_write_kernel");
}

// ---- few rows: 16 MT rows x 16 NT channels, eight wavefronts that share K block by block and read their operands from memory (a lane 32 values of a row's
// block, 16 g4 .. + 15 and 64 + 16 g4 .. + 15), the next block's in flight; the sums meet in LDS, in a fixed order.  FROM_X: rows of x are rounded on the way
// in, by every block for itself (a row's block of 128 is four lanes).
// A CU takes in the operands of 16 rows or channels (2 KB a block of K) in about 0.06 us, whatever is in flight: sixteen wavefronts, or three blocks each,
// take as long.  12 x 4096 x 4096 bf16: 6.4 us (the weights alone 3.4), 8.2 with x rounded on the way in.

template <typename T, int MT, int NT, bool FROM_X>
__global__ void __launch_bounds__(512)
linear_f8_few_kernel(LinearF8Args a) {
    constexpr int WV = 8, BM = 16 * MT, BN = 16 * NT, RS = BN + 4;      // wavefronts; RS: values of a row in LDS
    __shared__ __attribute__((aligned(16))) float s_sum[WV][BM * RS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g4 = lane >> 4;
    const int n0 = blockIdx.x * BN;
    const int64_t m0 = (int64_t)blockIdx.y * BM;
    const int KT = a.Kp / 128;                                          // blocks, dealt to the wavefronts in turn
    const uint8_t *wp[NT], *wsp[NT], *xp[MT], *xsp[MT];
    const T* xv[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        wp[j] = a.w8 + (int64_t)(n0 + 16 * j + col) * a.Kp + 16 * g4;  // (there are N rounded up to 256)
        wsp[j] = a.sw + 4 * (int64_t)(n0 + 16 * j + col);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t r = min(m0 + 16 * i + col, a.rows - 1);
        if constexpr (FROM_X) {
            xv[i] = (const T*)a.x + r * a.ldx;
        } else {
            xp[i] = a.x8 + r * a.Kp + 16 * g4;
            xsp[i] = a.sx + 4 * r;
        }
    }
    typedef typename AnyPiece<T>::type Any;
    f32x4 acc[MT][NT];
    i32x8 w[2][NT], x[FROM_X ? 1 : 2][MT];
    Raw8<T> raw[FROM_X ? 2 : 1][MT][4];
    int ws[2][NT], xs[FROM_X ? 1 : 2][MT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto operand = [&](const uint8_t* p) {
        const u32x4 lo = *reinterpret_cast<const u32x4*>(p), hi = *reinterpret_cast<const u32x4*>(p + 64);
        return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    auto load = [&](int set, int k) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            w[set][j] = operand(wp[j] + (int64_t)k * 128);
            ws[set][j] = wsp[j][f8_scale_at(a.Np, 0, k)];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if constexpr (FROM_X) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int at = 128 * k + 64 * (c >> 1) + 16 * g4 + 8 * (c & 1);
                    Raw8<T>& r = raw[set][i][c];
                    if (at + 8 <= a.K) {
#pragma unroll
                        for (int h = 0; h < (int)sizeof(T) / 2; ++h) r.w[h] = *reinterpret_cast<const Any*>(xv[i] + at + h * (16 / sizeof(T)));
                    } else {
                        T v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = at + e < a.K ? xv[i][at + e] : T(0);
                        __builtin_memcpy(&r, v, sizeof r);
                    }
                }
            } else {
                x[set][i] = operand(xp[i] + (int64_t)k * 128);
                xs[set][i] = xsp[i][f8_scale_at(a.rows, 0, k)];
            }
        }
    };
    auto mma = [&](int set) {
        const int from = FROM_X ? 0 : set;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if constexpr (FROM_X) {
                uint32_t m = 0;
#pragma unroll
                for (int c = 0; c < 4; ++c) m = largest8(m, raw[set][i][c]);
                const F8Scale z(max_32_apart(max_16_apart(m)));      // (of the lanes with the same number mod 16)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const q8_u32x2 p = z.pack8(raw[set][i][c]);
                    x[0][i][2 * c] = (int)p[0];
                    x[0][i][2 * c + 1] = (int)p[1];
                }
                xs[0][i] = (int)z.byte;
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if constexpr (sizeof(T) == 2) {
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[set][j], x[from][i], acc[i][j], 0, 0, 0, ws[set][j], 0, xs[from][i]);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f8_as_bf16(w[set][j], q, ws[set][j]), f8_as_bf16(x[from][i], q, xs[from][i]), acc[i][j], 0, 0, 0);
                }
            }
        }
    };
    // (each end has code of its own: where a load may or may not have been made, the wait in front of an instruction is for all of them)
    int k = wave, n = (KT - wave + WV - 1) / WV;            // next block, how many
    auto next = [&](int set) { load(set, k); k += WV; };
    if (n > 0) next(0);
    for (; n >= 3; n -= 2) { next(1); mma(0); next(0); mma(1); }
    if (n == 2) { next(1); mma(0); mma(1); }
    else if (n == 1) mma(0);
    // ---- the wavefronts' sums meet: the lane has row `col` of a tile and channels 4 g4 .. + 3
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(&s_sum[wave][(16 * i + col) * RS + 16 * j + 4 * g4]) = acc[i][j];
    __syncthreads();
    for (int idx = tid; idx < BM * BN / 4; idx += 64 * WV) {
        const int r = idx / (BN / 4), c = idx % (BN / 4) * 4, n = n0 + c;
        if (m0 + r >= a.rows || n >= a.N) continue;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WV; ++i) s += *reinterpret_cast<const f32x4*>(&s_sum[i][r * RS + c]);
        const f32x4 b = a.b ? *reinterpret_cast<const f32x4*>(a.b + n) : f32x4{0.f, 0.f, 0.f, 0.f};
        T* yp = (T*)a.y + (m0 + r) * a.N + n;
        const T* rp = (const T*)a.res + (m0 + r) * a.N + n;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= a.N) break;
            float v = s[e] + b[e];
            if (a.res) v += load1(rp + e);
            store1(yp + e, v);
        }
    }
}

template <typename T, int MT, int NT, bool FROM_X>
static int launch_few_as(const LinearF8Args& a, hipStream_t st) {
    linear_f8_few_kernel<T, MT, NT, FROM_X><<<dim3((unsigned)cdiv(a.N, 16 * NT), (unsigned)cdiv(a.rows, 16 * MT)), 512, 0, st>>>(a);
    return check_launch("linear_f8_few_kernel");
}
// Few rows rounded on the way in, by blocks of 16 x 16: every one reads and rounds all of its rows, but it is one launch and not two (2.4 us in a captured stream, 3 of the
// host's).  By rounds of 256 blocks and K; us in one / two launches: bf16 12 x 4096 x 4096 8.2 / 9.0, 64 x 1024 x 1024 4.8 / 6.4, 64 x 8192 x 1024 14.7 / 13.9, two rounds
// 12 x 1536 x 8192 7.4 / 8.2, 64 x 2048 x 2048 8.8 / 8.4; fp32 64 x 1024 x 1024 5.5 / 6.5, 12 x 2048 x 4096 7.6 / 7.7, 12 x 4096 x 4096 11.7 / 9.7, two rounds
// 64 x 512 x 2048 5.5 / 6.2
static bool few_from_x(int dtype, int64_t rows, int32_t K, int32_t N) {
    if (rows > 16384) return false;
    const int64_t rounds = cdiv(cdiv(rows, 16) * cdiv(N, 16), 256);
    const bool half = dtype == PSERVE_BF16;
    return rounds == 1 ? K <= (half ? 6144 : 2048) : rounds <= 4 && rounds * K <= (half ? 2560 : 1024);
}

// ---- many tiles: WGM x WGN wavefronts of 32 TM rows x 32 TN channels, a ring of NS stages of HB half blocks (64 of K) in LDS.
// A lane's operand of the 32 x 32 x 64 instruction is two 16-byte chunks of a row, chunks fh and 2 + fh of the half block's four (any order of K
// within a block does, the same for both operands).  The first operand's rows become the accumulators' rows, so the channels go
// first, in the order that leaves a lane with eight consecutive channels of one row of x.
__device__ __forceinline__ int lf_kperm(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

template <int WGM, int WGN, int TM, int TN, int HB, int NS>
struct LFCfg {
    static constexpr int NW = WGM * WGN, WM = 32 * TM, WN = 32 * TN, BM = WGM * WM, BN = WGN * WN;
    static constexpr int STAGE = (BM + BN) * 64 * HB;       // bytes
    static constexpr int LDS = NS * STAGE + 2 * 4 * (BM + BN) + 2 * 4 * BN;      // stages; scales of four blocks, of this group and the next; biases, of this tile and the next
    static constexpr int PRE = (NS * STAGE - 4096 * NW) / STAGE;    // stages beside the output staging (4 KB a wavefront at the ring's end)
    static_assert(PRE >= 1, "ring");
    static_assert(BM % (16 / HB * NW) == 0 && BN % (16 / HB * NW) == 0 && (BM + BN) % 64 == 0, "loads of a stage");
};

template <typename T, bool RES, int WGM, int WGN, int TM, int TN, int HB, int NS>
__global__ void __launch_bounds__(64 * WGM * WGN, 2)
linear_f8_tile_kernel(LinearF8Args a, int m_tiles, int total) {
    using Cfg = LFCfg<WGM, WGN, TM, TN, HB, NS>;
    constexpr int NW = Cfg::NW, WM = Cfg::WM, WN = Cfg::WN, BM = Cfg::BM, BN = Cfg::BN;
    constexpr int CH = 4 * HB, RP = 64 / CH * NW, A_LD = BM / RP, B_LD = BN / RP, LD = A_LD + B_LD, STAGE_V = Cfg::STAGE / 16;
    constexpr int S_LD = (BM + BN + 64 * NW - 1) / (64 * NW);
    constexpr bool ALONE = Cfg::LDS > 80 * 1024;            // a block a CU
    constexpr int GM = 4;                                   // row tiles of a group, see below
    extern __shared__ __attribute__((aligned(16))) uint8_t lf_smem[];
    u32x4* ring = reinterpret_cast<u32x4*>(lf_smem);        // [NS][rows of x, rows of w][CH chunks], swizzled: sixteen rows, all banks
    uint32_t* s_scale = reinterpret_cast<uint32_t*>(lf_smem + NS * Cfg::STAGE);      // [2][rows of x, rows of w] words of four blocks
    float* s_bias = reinterpret_cast<float*>(s_scale + 2 * (BM + BN));               // [2][channels]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WGM, wn = wave / WGM, fr = lane & 31, fh = lane >> 5;
    const int n_tiles = total / m_tiles, KT = a.Kp / 128, steps = KT * 2 / HB;

    // Tiles are numbered in groups of GM row tiles, rows fastest; XCD x (block id mod 8) takes the x-th eighth of the numbers, so
    // the blocks of an XCD run on neighbouring tiles and share the panels in its L2.
    const int xcd = blockIdx.x & 7, t_end = (int)((int64_t)total * (xcd + 1) / 8), t_step = gridDim.x >> 3;
    int t = (int)((int64_t)total * xcd / 8) + (blockIdx.x >> 3);
    if (t >= t_end) return;

    auto swizzle = [](int row) { return HB == 1 ? (row >> 2) & 3 : (row >> 1) & 7; };
    const int lr = 64 / CH * wave + lane / CH, gc = lane % CH ^ swizzle(lr);
    int a_off[A_LD], b_off[B_LD];                           // byte offsets from the tile's first row
    const uint8_t *a_base, *b_base, *s_base[S_LD];          // (s: scales of the thread's rows)
    int64_t m0 = 0;
    int n0 = 0;
    auto decode = [&](int tt) {
        const int grp = tt / (GM * n_tiles), r = tt - grp * (GM * n_tiles), gm = min(GM, m_tiles - grp * GM), nt = r / gm;
        m0 = (int64_t)(grp * GM + r - nt * gm) * BM;
        n0 = nt * BN;
    };
    auto setup = [&]() {
        a_base = a.x8 + m0 * a.Kp;
        b_base = a.w8 + (int64_t)n0 * a.Kp;
        const int last = (int)min((int64_t)BM, a.rows - m0) - 1, lastB = a.Np - 1 - n0;
#pragma unroll
        for (int l = 0; l < A_LD; ++l) a_off[l] = min(lr + l * RP, last) * a.Kp + gc * 16;
#pragma unroll
        for (int l = 0; l < B_LD; ++l) b_off[l] = min(lr + l * RP, lastB) * a.Kp + gc * 16;
#pragma unroll
        for (int l = 0; l < S_LD; ++l) {
            const int r = tid + l * 64 * NW;
            s_base[l] = r < BM ? a.sx + 4 * (m0 + min(r, last)) : a.sw + 4 * (int64_t)(n0 + min(r - BM, lastB));
        }
    };
    int odd = 0;                                            // half of the biases
    auto load_bias = [&](int half) {
#pragma unroll
        for (int c = 0; c < BN; c += 64 * NW)
            if (a.b && c + 64 * wave < BN)
                __builtin_amdgcn_global_load_lds((const void*)(a.b + min(n0 + c + tid, a.Np - 1)), (lds_void*)(s_bias + half * BN + c + 64 * wave), 4, 0, 0);
    };
    auto load_scales = [&](int group) {
#pragma unroll
        for (int l = 0; l < S_LD; ++l)
            if (64 * (wave + l * NW) < BM + BN)
                __builtin_amdgcn_global_load_lds((const void*)(s_base[l] + 4 * group * (64 * (wave + l * NW) < BM ? a.rows : (int64_t)a.Np)), (lds_void*)(s_scale + (group & 1) * (BM + BN) + 64 * (wave + l * NW)), 4, 0, 0);
    };
    // step h of 64 HB of K into stage st.  One load instruction a call, so that a refill is spread over the matrix instructions behind the barrier that frees
    // its stage
    auto load_one = [&](int h, int st, int l) {
        u32x4* dst = ring + st * STAGE_V + wave * 64;
        if (l < A_LD) __builtin_amdgcn_global_load_lds((const void*)(a_base + (int64_t)h * (64 * HB) + a_off[l < A_LD ? l : 0]), (lds_void*)(dst + l * (64 * NW)), 16, 0, 0);
        else __builtin_amdgcn_global_load_lds((const void*)(b_base + (int64_t)h * (64 * HB) + b_off[l >= A_LD ? l - A_LD : 0]),
                                              (lds_void*)(dst + BM * CH + (l - A_LD) * (64 * NW)), 16, 0, 0);
    };
    auto load_stage = [&](int h, int st) {
#pragma unroll
        for (int l = 0; l < LD; ++l) load_one(h, st, l);
    };
    const int rowA = wm * WM + fr, rowB = wn * WN + lf_kperm(fr);
    const u32x4 *pA[2 * HB], *pB[2 * HB];                   // the lane's chunks of a stage's first row tiles
#pragma unroll
    for (int c = 0; c < 2 * HB; ++c) {
        pA[c] = ring + rowA * CH + ((2 * c + fh) ^ swizzle(rowA));
        pB[c] = ring + (BM + rowB) * CH + ((2 * c + fh) ^ swizzle(rowB));
    }
    i32x8 fa[2][TM], fb[TN];
    auto fragment = [&](const u32x4* p, const u32x4* q, int at) {
        const u32x4 lo = p[at], hi = q[at];
        return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    };
    auto read_a = [&](int set, int st, int half, int i) { fa[set][i] = fragment(pA[2 * half], pA[2 * half + 1], st * STAGE_V + i * 32 * CH); };
    auto read_b = [&](int st, int half, int j) { fb[j] = fragment(pB[2 * half], pB[2 * half + 1], st * STAGE_V + j * 32 * CH); };
    int xa[TM], xb[TN], xa_next[TM], xb_next[TN];           // scale bytes of four blocks, and of the next four
    auto read_scales = [&](int group, int (&pa)[TM], int (&pb)[TN]) {
        const uint32_t* p = s_scale + (group & 1) * (BM + BN);
#pragma unroll
        for (int i = 0; i < TM; ++i) pa[i] = (int)p[rowA + 32 * i];
#pragma unroll
        for (int j = 0; j < TN; ++j) pb[j] = (int)p[BM + rowB + 32 * j];
    };
    auto mma = [&](int set, int i, int j, f32x16& c) {
        if constexpr (sizeof(T) == 2) {
            c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j], fa[set][i], c, 0, 0, 0, xb[j], 0, xa[i]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f8_as_bf16(fb[j], q, xb[j] & 255), f8_as_bf16(fa[set][i], q, xa[i] & 255), c, 0, 0, 0);
        }
        asm volatile("" : "+v"(c));                         // (it stays here: else the compiler sinks it past the branches around the loads)
    };
    constexpr int NM = TM * TN;                             // matrix instructions of half a block
    constexpr int SLOTS = HB == 1 ? NM - TM : 2 * NM - TM, LPS = (LD + SLOTS - 1) / SLOTS;      // of them with loads behind, loads behind one

    // Blocks in step, one a CU, all write their outputs at the same time, with the matrix cores idle, and multiply at the same time, with memory idle.  Where
    // the tiles do not come out even, the blocks that have one less therefore begin later, by about the time that an output takes (12,544 x 1536 x 6144 with
    // a residual 155 -> 149 us, x 4608 99 -> 91).
    const int share = t_end - (int)((int64_t)total * xcd / 8);          // tiles of the XCD
    if (ALONE && share > t_step && (int)(blockIdx.x >> 3) >= share % t_step && share % t_step != 0)
        for (int d = min(16, KT * 4 / 3); d > 0; --d) __builtin_amdgcn_s_sleep(16);      // 1024 cycles
    decode(t);
    setup();
    load_stage(0, 0);
    load_scales(0);
    load_bias(0);
    if (!a.b)
        for (int c = tid; c < 2 * BN; c += 64 * NW) s_bias[c] = 0.f;
#pragma unroll
    for (int st = 1; st < NS; ++st)
        if (st < steps) load_stage(st, st);
#pragma unroll 1
    for (;;) {
        f32x16 acc[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        if (steps >= NS) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 1) * LD) : "memory");       // the first step has landed
        else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int i = 0; i < TM; ++i) read_a(0, 0, 0, i);
#pragma unroll
        for (int j = 0; j < TN; ++j) read_b(0, 0, j);
        read_scales(0, xa, xb);
        int cur = 0;                                        // stage of this step
#pragma unroll 1
        for (int kt = 0; kt < KT; ++kt) {
            const bool turn = (kt & 3) == 3;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                // The step's last half: behind its first instructions every operand of the stage is read and the next step has landed (behind that are
                // the loads of those after it, where there are any; scales' loads among them only make the wait longer).  The stage is refilled behind
                // the instructions that follow, up to the next step's last half.  What is read behind the last step is not used
                const bool last = HB == 1 || ks == 1;
                const int h = HB == 1 ? 2 * kt + ks : kt, nxt = cur == NS - 1 ? 0 : cur + 1, prv = cur == 0 ? NS - 1 : cur - 1;
                const bool refill = h + NS < steps, late = h > 0 && h - 1 + NS < steps;
#pragma unroll
                for (int q = 0; q < NM; ++q) {
                    const int j = q / TM, i = q % TM;
                    mma(ks, i, j, acc[i][j]);
                    if (last) {
                        if (q == TM - 1) {
                            if (NS > 2 && h + NS <= steps) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((NS - 2) * LD) : "memory");
                            else asm volatile("s_waitcnt lgkmcnt(0)\n\ts_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
                        }
                        if (q >= TM - 1) {
                            if (q < 2 * TM - 1) read_a(ks ^ 1, nxt, 0, q - (TM - 1));
                            if (i == TM - 1) read_b(nxt, 0, j);
                            if (refill && q >= TM) {
#pragma unroll
                                for (int l = 0; l < LD; ++l) if (l / LPS == q - TM) load_one(h + NS, cur, l);
                            }
                        }
                    } else {
                        if (q < TM) read_a(1, cur, HB - 1, q);
                        if (i == TM - 1) read_b(cur, HB - 1, j);
                        if (late) {
#pragma unroll
                            for (int l = 0; l < LD; ++l) if (l / LPS == NM - TM + q) load_one(h - 1 + NS, prv, l);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (last) cur = nxt;
            }
            if ((kt & 3) == 0 && kt + 4 < KT) load_scales(kt / 4 + 1);
            if ((kt & 3) == 2) read_scales(kt / 4 + 1, xa_next, xb_next);       // (where there is a next group, two blocks later it has landed)
#pragma unroll
            for (int i = 0; i < TM; ++i) xa[i] = turn ? xa_next[i] : (int)((uint32_t)xa[i] >> 8);
#pragma unroll
            for (int j = 0; j < TN; ++j) xb[j] = turn ? xb_next[j] : (int)((uint32_t)xb[j] >> 8);
        }
        // ---- output in pieces of 32 rows x 128 bytes, through the end of the ring
        const int64_t r0 = m0 + wm * WM;
        const int c0 = n0 + wn * WN;
        constexpr int CV = 16 / sizeof(T), PC = 8 * CV;     // values of a 16-byte chunk, columns of a piece
        constexpr int PJ = PC / 32, NP = TN / PJ, PS = TM * NP, RQ = RES ? PS : 1;      // accumulator tiles of a piece; pieces of 32 rows, of all; those whose residuals are held
        static_assert(!RES || PS <= 4, "registers of the residuals");
        const int nt = t + t_step, er = lane >> 3, ec = lane & 7;
        // whole lines go past the L2, which holds the panels; where rows begin inside a line, its parts meet there
        const bool lines = a.N % (8 * CV) == 0 && !((uintptr_t)a.y & 127);
        typedef typename AnyPiece<T>::type Any;
        u32x4 rres[RQ][4];
        // the residual of piece p, eight whole lines an instruction
        auto res_load = [&](int p) {
            const int n = c0 + PC * (p % NP) + CV * ec;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t row = r0 + 32 * (p / NP) + 8 * k + er;
                const T* rp = (const T*)a.res + row * a.N + n;
                u32x4 v = {0, 0, 0, 0};
                if (row < a.rows) {
                    if (n + CV <= a.N) v = load_piece(rp, lines);
                    else if (n < a.N) {
                        T e[CV];
#pragma unroll
                        for (int c = 0; c < CV; ++c) e[c] = n + c < a.N ? rp[c] : T(0);
                        __builtin_memcpy(&v, e, sizeof v);
                    }
                }
                rres[p][k] = v;
            }
        };
        if constexpr (RES) {
#pragma unroll
            for (int p = 0; p < PS; ++p) res_load(p);
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // every wavefront has read its last fragments
        if (nt < t_end) {                                   // the first steps of the next tile come in beside the end of this one
            decode(nt);
            setup();
            load_stage(0, 0);
            load_scales(0);
            load_bias(odd ^ 1);
#pragma unroll
            for (int st = 1; st < Cfg::PRE; ++st)
                if (st < steps) load_stage(st, st);
        }
        const float* bias = s_bias + odd * BN + wn * WN + 8 * fh;
        u32x4* ep = ring + NS * STAGE_V - NW * 256 + wave * 256;        // [32 rows][8 chunks], chunk ^ ((row >> 1) & 7)
        const int sw = (fr >> 1) & 7;
        // chunk of the lane's 16-byte word q of a piece: words 2 jj + c (bf16), 2 c + h (fp32)
        auto chunk = [&](int q) { return (sizeof(T) == 2 ? 2 * q + fh : 4 * (q >> 1) + 2 * fh + (q & 1)) ^ sw; };
#pragma unroll
        for (int p = 0; p < PS; ++p) {
            const int i = p / NP, jp = p % NP, pcol = c0 + PC * jp;
            if (pcol >= a.N) continue;
            u32x4 beside[4];
            if constexpr (RES) {                            // the residual as the accumulators lie, through the staging
#pragma unroll
                for (int k = 0; k < 4; ++k) ep[(8 * k + er) * 8 + (ec ^ (((8 * k + er) >> 1) & 7))] = rres[p][k];
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int q = 0; q < 4; ++q) beside[q] = ep[fr * 8 + chunk(q)];
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll
            for (int jj = 0; jj < PJ; ++jj)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float v[8], b[8];
                    load8(bias + PC * jp + 32 * jj + 16 * c, b);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[e] = acc[i][jp * PJ + jj][8 * c + e] + b[e];
                        if constexpr (RES && sizeof(T) == 2) {
                            const uint32_t r = beside[2 * jj + c][e / 2];
                            v[e] += e & 1 ? __uint_as_float(r & 0xffff0000u) : __uint_as_float(r << 16);
                        } else if constexpr (RES) {
                            v[e] += __uint_as_float(beside[2 * c + e / 4][e % 4]);
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
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int rr = 8 * k + er, n = pcol + CV * ec;
                const int64_t row = r0 + 32 * i + rr;
                const u32x4 o = ep[rr * 8 + (ec ^ ((rr >> 1) & 7))];
                T* yp = (T*)a.y + row * a.N + n;
                if (row < a.rows && n + CV <= a.N) {
                    store_piece(yp, o, lines);
                } else if (row < a.rows) {
                    T e[CV];
                    __builtin_memcpy(e, &o, sizeof o);
#pragma unroll
                    for (int c = 0; c < CV; ++c)
                        if (n + c < a.N) yp[c] = e[c];
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (nt >= t_end) break;
        t = nt;
        odd ^= 1;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // the staging is done with
#pragma unroll
        for (int st = Cfg::PRE; st < NS; ++st)
            if (st < steps) load_stage(st, st);
    }
}

template <typename T, bool RES, int WGM, int WGN, int TM, int TN, int HB, int NS>
static int launch_tile_as(const LinearF8Args& a, hipStream_t st) {
    using Cfg = LFCfg<WGM, WGN, TM, TN, HB, NS>;
    PS_SET_LDS_ONCE((linear_f8_tile_kernel<T, RES, WGM, WGN, TM, TN, HB, NS>), Cfg::LDS);
    const int64_t mt = cdiv(a.rows, Cfg::BM), total = mt * cdiv(a.N, Cfg::BN);
    const unsigned grid = (unsigned)(8 * cdiv(std::min<int64_t>(total, Cfg::LDS > 80 * 1024 ? 256 : 512), 8));
    linear_f8_tile_kernel<T, RES, WGM, WGN, TM, TN, HB, NS><<<grid, 64 * Cfg::NW, Cfg::LDS, st>>>(a, (int)mt, (int)total);
    return check_launch("linear_f8_tile_kernel");
}
// The kernel with the least time by its rounds, us of a launch in a captured stream.
// Blocks of few rows, 256 at once: so much for each 16 rows of operands and block of K (measured at K = 8192, 256 blocks of 16 x 16 / 16 x 32 / 32 x 32:
// 10.4 / 15.1 / 18.5, K = 1536 3.8 / 4.7 / 5.3).  Tiles: 256 at once of the largest, 512 of the others, of which the last round's are alone
// on their CUs; so much for each block of K and so much for its beginning and end, fitted to (256 x 256 / 128 x 128 / 64 x 128 us, bf16) 12,544 x 1536 x 6144
// with a residual 158 / 164 / 197, 12,544 x 6144 x 1536 with one 164 / 144 / 177, 2048 x 4096 x 4096 46 / 36 / 45, 3000 x 3000 x 3000 37 / 43 / 41, 2048 x 2048 x 2048
// 29 / 17 / 14, 100 x 2048 x 8192 25 / 13 / 9, 6000 x 1000 x 3000 with a residual 53 / 40 / 43; fp32: 8000 x 500 x 1500 with one 64 / 37 / 36 (the largest
// tile's operands spill there, and it is left out), 500 x 3000 x 2000 68 / 26 / 19.  Tiles against few rows: 256 x 512 x 1024 5.1 / 3.7, 64 x 8192 x 1024 25 / 15,
// 33 x 4096 x 4096 14.6 / 11, 200 x 4096 x 4096 15 / 32
enum { LF_FROM_X = 1, LF_FEW_16_16 = 11, LF_FEW_16_32 = 12, LF_FEW_32_32 = 22, LF_TILES_64 = 64, LF_TILES_128 = 128, LF_TILES_256 = 256 };      // (few: groups of 16 rows, of 16 channels)
static int product_form(bool half, bool res, int64_t rows, int32_t K, int32_t N) {
    const double KT = f8_width(K) / 128;
    auto few = [&](int mt, int nt) {
        const int64_t blocks = cdiv(rows, 16 * mt) * cdiv(N, 16 * nt);
        return blocks > 2048 ? 1e9 : 2.4 + (double)cdiv(blocks, 256) * (0.0625 * (mt + nt) * KT + (half ? 0.3 : 0.5));
    };
    auto tiles = [&](int bm, int bn, int at_once, double step, double ends) {
        const int64_t total = cdiv(rows, bm) * cdiv(N, bn), rest = total % at_once;
        const double last = rest == 0 ? 0.0 : at_once == 256 ? 1.0 : 0.55 + 0.45 * (double)rest / at_once;
        return ((double)(total / at_once) + last) * (step * KT + ends);
    };
    const double small = half ? tiles(64, 128, 512, 0.64, res ? 4.5 : 4.0) : tiles(64, 128, 512, 1.05, 7.5);
    const double mid = half ? tiles(128, 128, 512, 1.06, res ? 6.0 : 5.0) : tiles(128, 128, 512, 1.85, 13.0);
    const double large = half ? tiles(256, 256, 256, 1.5, res ? 14.0 : 11.0) : 1e9;
    const double f11 = few(1, 1), f12 = few(1, 2), f22 = few(2, 2);
    if (std::min(f11, std::min(f12, f22)) < std::min(small, std::min(mid, large)) + (half ? 1.3 : 0.0))      // (a launch of few bf16 tiles takes 1.3 more than the fit says)
        return f11 <= f12 && f11 <= f22 ? LF_FEW_16_16 : f12 <= f22 ? LF_FEW_16_32 : LF_FEW_32_32;
    if (half && large <= std::min(mid, small)) return LF_TILES_256;
    return mid <= small ? LF_TILES_128 : LF_TILES_64;
}

template <typename T, bool RES>
static int launch_product(const LinearF8Args& a, hipStream_t st) {
    const int form = product_form(sizeof(T) == 2, RES, a.rows, a.K, a.N);
    if constexpr (sizeof(T) == 2)
        if (form == LF_TILES_256) return launch_tile_as<T, RES, 4, 2, 2, 4, 1, 4>(a, st);
    switch (form) {
        case LF_FEW_16_16: return launch_few_as<T, 1, 1, false>(a, st);
        case LF_FEW_16_32: return launch_few_as<T, 1, 2, false>(a, st);
        case LF_FEW_32_32: return launch_few_as<T, 2, 2, false>(a, st);
        case LF_TILES_128: return launch_tile_as<T, RES, 2, 2, 2, 2, 2, 2>(a, st);
        default: return launch_tile_as<T, RES, 2, 2, 1, 2, 2, 3>(a, st);
    }
}

template <typename T>
static int forward(LinearF8Args a, hipStream_t st) {
    if (a.x) {
        if (few_from_x(sizeof(T) == 2 ? PSERVE_BF16 : PSERVE_F32, a.rows, a.K, a.N)) return launch_few_as<T, 1, 1, true>(a, st);
        PS_TRY(launch_rows_write<T>(a.x, a.ldx, a.rows, a.K, a.x8, a.sx, st));
    }
    return a.res ? launch_product<T, true>(a, st) : launch_product<T, false>(a, st);
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
    if (rows8) {
        a.x8 = (uint8_t*)rows8;
        a.sx = a.x8 + (size_t)a.rows * op->Kp;
    }
    a.res = residual; a.y = y;
    a.w8 = op->w; a.sw = op->scale; a.b = op->b;
    a.K = op->K; a.N = op->N; a.Kp = op->Kp; a.Np = op->Np;
    return op->dtype == PSERVE_BF16 ? forward<uint16_t>(a, st) : forward<float>(a, st);
}

}  // namespace pserve

extern "C" {

// For tests (not in the header): the form of the product that a call takes, see LF_FROM_X ..
int pserve_test_linear_f8_form(int dtype, int64_t rows, int32_t K, int32_t N, int from_x, int residual) {
    return from_x && few_from_x(dtype, rows, K, N) ? LF_FROM_X : product_form(dtype == PSERVE_BF16, residual != 0, rows, K, N);
}

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
        op->Kp = f8_width(K); op->Np = (int32_t)cdiv(N, 256) * 256;
        PS_CHECK_HIP(hipGetDevice(&op->device));
        hipStream_t st = (hipStream_t)stream;
        PS_TRY(op->pool.alloc((void**)&op->w, (size_t)op->Np * op->Kp));
        const size_t scales = (size_t)op->Np * f8_scales(K);
        PS_TRY(op->pool.alloc((void**)&op->scale, scales));
        PS_CHECK_HIP(hipMemsetAsync(op->scale, 127, scales, st));
        const dim3 grid(op->Np / 64, op->Kp / 128);
        if (dtype == PSERVE_BF16) linear_f8_pack_kernel<<<grid, 256, 0, st>>>((const uint16_t*)w, K, N, op->Kp, op->Np, op->w, op->scale);
        else linear_f8_pack_kernel<<<grid, 256, 0, st>>>((const float*)w, K, N, op->Kp, op->Np, op->w, op->scale);
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
    *bytes = few_from_x(op->dtype, rows, op->K, op->N) ? 0 : f8_bytes(rows, op->K);
    return PSERVE_OK;
}

int pserve_linear_f8_forward(const pserve_linear_f8_t* op, const void* x, int64_t ldx, int64_t rows, const void* residual, void* workspace,
                             size_t workspace_bytes, void* y, void* stream) {
    static const char who[] = "pserve_linear_f8_forward";
    PS_REQUIRE(op, "%s: NULL argument", who);
    size_t need = 0;
    PS_TRY(pserve_linear_f8_workspace(op, rows, &need));
    if (rows == 0) return PSERVE_OK;
    PS_REQUIRE(x && y && (workspace || need == 0), "%s: NULL buffer", who);
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
