// Linear layers in 8-bit integers (pserve_linear8_*), gfx950.
//
//   y[t][n] = (sum_k qx[t][k] qw[n][k]) * (sx[t] * sw[n]) + b[n] + residual[t][n]
//
// Two launches: the rows of x are quantised into the workspace (one pass over x, bound by memory), then the product runs on
// v_mfma_i32_32x32x32_i8, twice the rate of bf16.  Sums are exact in 32 bits: 127^2 * 131072 < 2^31.
// qw is kept as [N rounded up to 256][K rounded up to 128], qx as [rows][K rounded up to 128], both filled up with zeros, so a step
// of K is a row of 128 bytes in eight chunks, whatever K and N are; only the stores look at N.
// Measured: 8192 x 8192 x 8192 524 us, 2.1 POPS, which the power limit holds (2.7 with zeros); 12,544 x 1536 x 6144 with a residual, bf16, 17 us
// for the rows (58 MB) and 140 .. 144 for the product; 12 x 4096 x 4096 4.6 and 6.5 (17 MB).  fp32 layers with a residual and an N that is
// no multiple of 4 spill 87 registers in the largest tiles: 4096 x 1024 x 4099 135 us, x 4100 79.
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

// ---- rows of x: TPR threads a row, CH chunks of eight values a thread in registers; chunks behind those are read twice.
// A wavefront a row needs no barrier and, from a few hundred rows on, fills the chip; fewer rows take a block each.
template <typename T, int TPR, int CH, bool VEC>
__global__ void __launch_bounds__(256)
linear8_rows_kernel(Linear8Args a) {
    __shared__ uint32_t s_max[4];
    const int t = threadIdx.x % TPR;
    const int64_t row = block_of_lines() * (256 / TPR) + threadIdx.x / TPR;
    if (TPR < 256 && row >= a.rows) return;
    const T* x = (const T*)a.x + row * a.ldx;
    typedef Raw8<T> Chunk;
    constexpr int W = sizeof(T) / 2;                        // 16-byte words of a chunk
    auto get = [&](int c) -> Chunk {
        Chunk r;
        if (VEC) {
#pragma unroll
            for (int i = 0; i < W; ++i) r.w[i] = 8 * c < a.K ? *reinterpret_cast<const u32x4*>(x + 8 * c + i * (8 / W)) : u32x4{0, 0, 0, 0};
        } else {
            T v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 8 * c + i < a.K ? x[8 * c + i] : T(0);
            __builtin_memcpy(&r, v, sizeof r);
        }
        return r;
    };
    const int chunks = a.Kp / 8;
    Chunk held[CH];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) held[i] = get(t + i * TPR);
#pragma unroll
    for (int i = 0; i < CH; ++i) m = largest8(m, held[i]);
    for (int c = t + CH * TPR; c < chunks; c += TPR) m = largest8(m, get(c));
    m = lanes_max<64>(m);
    if (TPR == 256) {
        if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
        __syncthreads();
        m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    }
    const Quant8 z(m);
    if (t == 0) a.x_scale[row] = z.scale;
    int8_t* o = a.x8 + row * a.Kp;
    auto put = [&](int c, const Chunk& r) {
        float v[8];
        values8(r, v);
        *reinterpret_cast<q8_u32x2*>(o + 8 * c) = pack8(z, v);
    };
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (t + i * TPR < chunks) put(t + i * TPR, held[i]);
    for (int c = t + CH * TPR; c < chunks; c += TPR) put(c, get(c));
}

template <typename T, bool VEC>
static int launch_rows_as(const Linear8Args& a, hipStream_t st) {
    if (a.rows < 512 && a.Kp > 512) linear8_rows_kernel<T, 256, 4, VEC><<<(unsigned)a.rows, 256, 0, st>>>(a);
    else if (a.Kp <= 1024) linear8_rows_kernel<T, 64, 2, VEC><<<block_lines(cdiv(a.rows, 4)), 256, 0, st>>>(a);
    else if (a.Kp <= 2048) linear8_rows_kernel<T, 64, 4, VEC><<<block_lines(cdiv(a.rows, 4)), 256, 0, st>>>(a);
    else linear8_rows_kernel<T, 64, 8, VEC><<<block_lines(cdiv(a.rows, 4)), 256, 0, st>>>(a);
    return check_launch("linear8_rows_kernel");
}
template <typename T>
static bool rows_vec(const Linear8Args& a) { return a.K % 8 == 0 && a.ldx % (16 / sizeof(T)) == 0 && !((uintptr_t)a.x & 15); }
template <typename T>
static int launch_rows(const Linear8Args& a, hipStream_t st) {
    return rows_vec<T>(a) ? launch_rows_as<T, true>(a, st) : launch_rows_as<T, false>(a, st);
}

// ---- the product: WGM x WGN wavefronts of 32 TM rows x 32 TN channels, two stages of 128 values of K
__device__ __forceinline__ int l8_kperm(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }   // as in the bf16 layers

template <int WGM, int WGN, int TM, int TN>
struct L8Cfg {
    static constexpr int NW = WGM * WGN, WM = 32 * TM, WN = 32 * TN, BM = WGM * WM, BN = WGN * WN;
    static constexpr int STAGE = (BM + BN) * 128;           // bytes
    static constexpr int LDS = 2 * STAGE + 2 * 2 * BN * 4;  // ring; scales and biases of a tile's channels, of this tile and the next
    static_assert(STAGE >= NW * 4096, "the output staging (4 KB a wavefront) reuses a stage");
};

// The accumulators of a lane are eight consecutive channels of one row (kperm), so a piece of 32 rows x 128 bytes passes LDS in 16-byte
// pieces and leaves in stores of whole 128-byte lines.
// VEC: rows of y and of the residual lie on the 16-byte grid.
template <typename T, bool RES, bool VEC, int WGM, int WGN, int TM, int TN>
__global__ void __launch_bounds__(64 * WGM * WGN, 2)
linear8_tile_kernel(Linear8Args a, int m_tiles, int total) {
    using Cfg = L8Cfg<WGM, WGN, TM, TN>;
    constexpr int NW = Cfg::NW, WM = Cfg::WM, WN = Cfg::WN, BM = Cfg::BM, BN = Cfg::BN;
    constexpr int RP = 8 * NW, A_LD = BM / RP, B_LD = BN / RP, LD = A_LD + B_LD, STAGE_V = Cfg::STAGE / 16;
    constexpr int GM = 8;                                   // row tiles of a group, see below
    extern __shared__ __attribute__((aligned(16))) uint8_t l8_smem[];
    float* s_cols = reinterpret_cast<float*>(l8_smem + 2 * Cfg::STAGE);
    u32x4* ring = reinterpret_cast<u32x4*>(l8_smem);        // [2][rows of x, rows of w][8 chunks], chunk ^ ((row >> 1) & 7)
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
    const int8_t *a_base, *b_base;
    int64_t m0 = 0;
    int n0 = 0;
    auto decode = [&](int tt) {
        const int grp = tt / (GM * n_tiles), r = tt - grp * (GM * n_tiles), gm = min(GM, m_tiles - grp * GM), nt = r / gm;
        m0 = (int64_t)(grp * GM + r - nt * gm) * BM;
        n0 = nt * BN;
    };
    int buf = 0;
    auto setup = [&](int to) {
        a_base = a.x8 + m0 * a.Kp;
        b_base = a.w8 + (int64_t)n0 * a.Kp;
        const int last = (int)min((int64_t)BM, a.rows - m0) - 1;
#pragma unroll
        for (int l = 0; l < A_LD; ++l) a_off[l] = min(lr + l * RP, last) * a.Kp + gc * 16;
#pragma unroll
        for (int l = 0; l < B_LD; ++l) b_off[l] = min(lr + l * RP, a.Np - 1 - n0) * a.Kp + gc * 16;
        for (int c = tid; c < BN; c += 64 * NW) {           // (both are filled up to Np)
            const int n = min(n0 + c, a.Np - 1);
            s_cols[to * 2 * BN + c] = a.w_scale[n];
            s_cols[to * 2 * BN + BN + c] = a.b ? a.b[n] : 0.f;
        }
    };
    auto load_stage = [&](int kt, int stage) {
        u32x4* dst = ring + stage * STAGE_V + wave * 64;
        const int8_t *ap = a_base + (int64_t)kt * 128, *bp = b_base + (int64_t)kt * 128;
#pragma unroll
        for (int l = 0; l < A_LD; ++l) __builtin_amdgcn_global_load_lds((const void*)(ap + a_off[l]), (lds_void*)(dst + l * (64 * NW)), 16, 0, 0);
#pragma unroll
        for (int l = 0; l < B_LD; ++l) __builtin_amdgcn_global_load_lds((const void*)(bp + b_off[l]), (lds_void*)(dst + BM * 8 + l * (64 * NW)), 16, 0, 0);
    };
    const int rowA = wm * WM + fr, rowB = wn * WN + l8_kperm(fr);
    const u32x4 *pA = ring + rowA * 8, *pB = ring + BM * 8 + rowB * 8;
    const int swA = (rowA >> 1) & 7, swB = (rowB >> 1) & 7;

    // One load instruction a call, so that the refill of a stage is spread over the matrix instructions behind the barrier that frees
    // it: the wavefronts' loads in one burst queue at the address unit and hold what stands behind them.
    auto load_one = [&](int kt, int stage, int l) {
        u32x4* dst = ring + stage * STAGE_V + wave * 64;
        if (l < A_LD) __builtin_amdgcn_global_load_lds((const void*)(a_base + (int64_t)kt * 128 + a_off[l < A_LD ? l : 0]), (lds_void*)(dst + l * (64 * NW)), 16, 0, 0);
        else __builtin_amdgcn_global_load_lds((const void*)(b_base + (int64_t)kt * 128 + b_off[l >= A_LD ? l - A_LD : 0]),
                                              (lds_void*)(dst + BM * 8 + (l - A_LD) * (64 * NW)), 16, 0, 0);
    };
    constexpr int NM = TM * TN, NR = TM + TN, QB = NM - NR < 2 ? NM - NR : 2;   // MFMAs, fragment reads of a sub-step; MFMAs in front of the barrier
    constexpr int SP = NM >= 8 ? 2 : 1;                     // MFMAs between two loads
    static_assert(QB >= 0 && LD * SP <= NM - QB + 3 * NM, "loads of a step");
    i32x4 fa[2][TM], fb[2][TN];
    // fragment r of sub-step ks: a row tile first, the channel tiles, the other row tiles
    auto read = [&](int set, int stage, int ks, int r) {
        const u32x4 *sA = pA + stage * STAGE_V, *sB = pB + stage * STAGE_V;
        const int c = 2 * ks + fh;
        if (r == 0) fa[set][0] = __builtin_bit_cast(i32x4, sA[c ^ swA]);
        else if (r <= TN) fb[set][r - 1] = __builtin_bit_cast(i32x4, sB[(r - 1) * 256 + (c ^ swB)]);
        else fa[set][r - TN] = __builtin_bit_cast(i32x4, sA[(r - TN) * 256 + (c ^ swA)]);
    };

    decode(t);
    setup(0);
    load_stage(0, 0);
    if (KT > 1) load_stage(1, 1);
#pragma unroll 1
    for (;;) {
        i32x16 acc[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
        if (KT > 1) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(LD) : "memory");    // the first step has landed
        else asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int r = 0; r < NR; ++r) read(0, 0, 0, r);
#pragma unroll 1
        for (int kt = 0; kt < KT; ++kt) {
            const int cur = kt & 1, nxt = cur ^ 1;
            const bool refill = kt + 2 < KT, late = kt > 0 && kt + 1 < KT;      // loads into `cur` behind the barrier; the rest of the step before's
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int q = 0; q < NM; ++q) {
                    const int i = q / TN, j = q % TN, f = ks & 1;
                    // every fragment of this step is read (its stage is free) and the next step has landed
                    if (ks == 3 && q == QB) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[f][j], fa[f][i], acc[i][j], 0, 0, 0);
                    const int r = ks == 3 ? q - QB : q;
                    if (r >= 0 && r < NR) {
                        if (ks < 3) read(f ^ 1, cur, ks + 1, r);
                        else read(f ^ 1, nxt, 0, r);
                    }
                    const int sl = ks == 3 ? q - QB : NM - QB + ks * NM + q;    // place behind the barrier
                    if (ks == 3 && q >= QB && refill) {
#pragma unroll
                        for (int l = 0; l < LD; ++l) if (l * SP == sl) load_one(kt + 2, cur, l);
                    }
                    if (ks < 3 && late) {
#pragma unroll
                        for (int l = 0; l < LD; ++l) if (l * SP == sl) load_one(kt + 1, nxt, l);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
        }
        // ---- output in pieces of 32 rows x 128 bytes, through the second stage
        const int64_t r0 = m0 + wm * WM;
        const int c0 = n0 + wn * WN;
        constexpr int CV = 16 / sizeof(T), PC = 8 * CV;     // values of a 16-byte chunk, columns of a piece
        constexpr int PJ = PC / 32, NP = TN / PJ;           // accumulator tiles of a piece, pieces of 32 rows
        const int nt = t + t_step;
        u32x4 rres[RES ? 2 : 1][4];
        // the lane's residual of piece p: row fr of the piece, chunks in the accumulators' order
        auto res_load = [&](int p) {
            const int64_t row = min(r0 + 32 * (p / NP) + fr, a.rows - 1);
            const T* rp = (const T*)a.res + row * a.N;
            const int c = c0 + PC * (p % NP) + 8 * fh;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int at = sizeof(T) == 2 ? c + 16 * q : c + 16 * (q >> 1) + 4 * (q & 1);
                rres[p & 1][q] = *reinterpret_cast<const u32x4*>(rp + (at < a.N ? at : 0));
            }
        };
        if constexpr (RES && VEC) res_load(0);
        float sx[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) sx[i] = a.x_scale[min(r0 + 32 * i + fr, a.rows - 1)];
        const float* cs = s_cols + buf * 2 * BN + wn * WN + 8 * fh;             // scales of the lane's channels; the biases BN further
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // every wavefront has read its last fragments
        if (nt < t_end) {                                   // the first step of the next tile comes in beside the end of this one
            decode(nt);
            setup(buf ^ 1);
            load_stage(0, 0);
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
            if constexpr (RES && VEC) if (p + 1 < TM * NP) res_load(p + 1);
            if (pcol >= a.N) continue;
            const bool in = pcol + lane % PC < a.N;
            if constexpr (RES && !VEC) {                    // whole rows in, a value a lane
                T v[32 / RI];
#pragma unroll
                for (int r = 0; r < 32 / RI; ++r) {
                    const int64_t row = r0 + 32 * i + lane / PC + r * RI;
                    v[r] = in && row < a.rows ? ((const T*)a.res)[row * a.N + pcol + lane % PC] : T(0);
                }
#pragma unroll
                for (int r = 0; r < 32 / RI; ++r) *cell(lane / PC + r * RI) = v[r];
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int q = 0; q < 4; ++q) rres[p & 1][q] = ep[fr * 8 + chunk(q)];
                __builtin_amdgcn_wave_barrier();
            }
#pragma unroll
            for (int jj = 0; jj < PJ; ++jj)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float* sp = cs + PC * jp + 32 * jj + 16 * c;
                    float v[8], w[8], b[8];
                    load8(sp, w);
                    load8(sp + BN, b);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[e] = (float)acc[i][jp * PJ + jj][8 * c + e] * (sx[i] * w[e]) + b[e];
                        if constexpr (RES && sizeof(T) == 2) {
                            const uint32_t r = rres[p & 1][2 * jj + c][e / 2];
                            v[e] += e & 1 ? __uint_as_float(r & 0xffff0000u) : __uint_as_float(r << 16);
                        } else if constexpr (RES) {
                            v[e] += __uint_as_float(rres[p & 1][2 * c + e / 4][e % 4]);
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
        buf ^= 1;
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // the staging is done with
        if (KT > 1) load_stage(1, 1);
    }
}

template <typename T, bool RES, bool VEC, int WGM, int WGN, int TM, int TN>
static int launch_tile_as(const Linear8Args& a, hipStream_t st) {
    using Cfg = L8Cfg<WGM, WGN, TM, TN>;
    PS_SET_LDS_ONCE((linear8_tile_kernel<T, RES, VEC, WGM, WGN, TM, TN>), Cfg::LDS);
    const int64_t mt = cdiv(a.rows, Cfg::BM), total = mt * cdiv(a.N, Cfg::BN);
    const unsigned grid = (unsigned)(8 * cdiv(std::min<int64_t>(total, Cfg::LDS > 80 * 1024 ? 256 : 512), 8));
    linear8_tile_kernel<T, RES, VEC, WGM, WGN, TM, TN><<<grid, 64 * Cfg::NW, Cfg::LDS, st>>>(a, (int)mt, (int)total);
    return check_launch("linear8_tile_kernel");
}

// ---- few rows or few tiles: 16 MT rows x 16 NT channels, eight wavefronts that share K and read their operands from memory in the layout
// of v_mfma_i32_16x16x64_i8 (16 rows x 64 bytes a load), the next step's in flight; the sums meet in LDS.  Quantising the rows of x in
// here as well, in one launch, took 21 .. 25 us for 1 .. 12 rows x 4096 x 4096 where the two launches take 9 .. 10: every block of
// channels does it again.
template <typename T, int MT, int NT>
__global__ void __launch_bounds__(512)
linear8_few_kernel(Linear8Args a, int m_tiles) {
    constexpr int BM = 16 * MT, BN = 16 * NT, RS = BN + 4, WV = 8;      // RS: ints of a row in LDS
    __shared__ __attribute__((aligned(16))) int32_t s_sum[WV][BM * RS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, g4 = lane >> 4;
    const int64_t m0 = (int64_t)(blockIdx.x % m_tiles) * BM;
    const int n0 = (int)(blockIdx.x / m_tiles) * BN;
    const int KT = a.Kp / 64;                                           // steps, dealt to the wavefronts in shares
    const int per = (KT + WV - 1) / WV, k0 = min(KT, wave * per), k1 = min(KT, k0 + per);
    const int8_t *wp[NT], *xp[MT];
#pragma unroll
    for (int j = 0; j < NT; ++j) wp[j] = a.w8 + (int64_t)min(n0 + 16 * j + col, a.Np - 1) * a.Kp + 16 * g4;
#pragma unroll
    for (int i = 0; i < MT; ++i) xp[i] = a.x8 + min(m0 + 16 * i + col, a.rows - 1) * a.Kp + 16 * g4;
    i32x4 acc[MT][NT], w[2][NT], x[2][MT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
    auto load = [&](int set, int k) {
        k = min(k, KT - 1);
#pragma unroll
        for (int j = 0; j < NT; ++j) w[set][j] = *reinterpret_cast<const i32x4*>(wp[j] + (int64_t)k * 64);
#pragma unroll
        for (int i = 0; i < MT; ++i) x[set][i] = *reinterpret_cast<const i32x4*>(xp[i] + (int64_t)k * 64);
    };
    auto mma = [&](int set) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[set][j], x[set][i], acc[i][j], 0, 0, 0);
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
        for (int j = 0; j < NT; ++j) *reinterpret_cast<i32x4*>(&s_sum[wave][(16 * i + col) * RS + 16 * j + 4 * g4]) = acc[i][j];
    __syncthreads();
    for (int idx = tid; idx < BM * BN / 4; idx += 64 * WV) {
        const int r = idx / (BN / 4), c = idx % (BN / 4) * 4, n = n0 + c;
        const int64_t row = m0 + r;
        if (row >= a.rows || n >= a.N) continue;
        i32x4 s = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < WV; ++i) s += *reinterpret_cast<const i32x4*>(&s_sum[i][r * RS + c]);
        const float sx = a.x_scale[row];
        const f32x4 sw = *reinterpret_cast<const f32x4*>(a.w_scale + n);
        const f32x4 b = a.b ? *reinterpret_cast<const f32x4*>(a.b + n) : f32x4{0.f, 0.f, 0.f, 0.f};
        T* yp = (T*)a.y + row * a.N + n;
        const T* rp = (const T*)a.res + row * a.N + n;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= a.N) break;
            float v = (float)s[e] * (sx * sw[e]) + b[e];
            if (a.res) v += load1(rp + e);
            store1(yp + e, v);
        }
    }
}

template <typename T, int MT, int NT>
static int launch_few(const Linear8Args& a, hipStream_t st) {
    const int64_t mt = cdiv(a.rows, 16 * MT);
    linear8_few_kernel<T, MT, NT><<<(unsigned)(mt * cdiv(a.N, 16 * NT)), 512, 0, st>>>(a, (int)mt);
    return check_launch("linear8_few_kernel");
}

template <typename T, bool RES, bool VEC>
static int launch_tile_vec(const Linear8Args& a, hipStream_t st) {
    // (a tile a CU: 12,544 x 1536 x 6144 179 us with 128 x 128 tiles, 156 with these)
    if (cdiv(a.rows, 256) * cdiv(a.N, 256) >= 256) return launch_tile_as<T, RES, VEC, 4, 2, 2, 4>(a, st);
    return launch_tile_as<T, RES, VEC, 2, 2, 2, 2>(a, st);
}
template <typename T>
static int launch_tile(const Linear8Args& a, hipStream_t st) {
    const bool vec = a.N % (16 / sizeof(T)) == 0 && !(((uintptr_t)a.y | (uintptr_t)a.res) & 15);
    if (a.res) return vec ? launch_tile_vec<T, true, true>(a, st) : launch_tile_vec<T, true, false>(a, st);
    return vec ? launch_tile_vec<T, false, true>(a, st) : launch_tile_vec<T, false, false>(a, st);
}

template <typename T>
static int forward(const Linear8Args& a, hipStream_t st) {
    PS_TRY(launch_rows<T>(a, st));
    // us of both launches, 16 x 16 / 32 x 32 / 128 x 128 tiles: 12 x 4096 x 4096 10.1 / 12.7 / 24.4, 32 x 4096 x 4096 14.4 / 14.3 / 24.8,
    // 64 x 4096 x 4096 22.6 / 15.9 / 25.7, 200 x 2048 x 2048 20.5 / 14.9 / 17.6, 500 x 1280 x 1280 (40 tiles) 18.5 / 14.0 / 14.6,
    // 256 x 1280 x 5120 (80 tiles) 31.4 / 21.0 / 14.5
    if (a.rows <= 32) return launch_few<T, 1, 1>(a, st);
    if (cdiv(a.rows, 128) * cdiv(a.N, 128) <= 64) return launch_few<T, 2, 2>(a, st);
    return launch_tile<T>(a, st);
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
    PS_REQUIRE(rows >= 0 && rows < (1 << 26), "pserve_linear8: %lld rows (fewer than 2^26)", (long long)rows);
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
    return op->dtype == PSERVE_BF16 ? forward<uint16_t>(a, st) : forward<float>(a, st);
}

}  // extern "C"
