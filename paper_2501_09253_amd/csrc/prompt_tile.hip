// Causal attention with grouped heads, gfx950: bf16, tiles of 128 or 256 rows on the 32 x 32 x 16 matrix instructions.
//
// A row is a query token's head; the G heads of a key/value head are neighbouring rows, so the 256 rows of a block are
// 256 / G tokens: keys and values are staged once for all of them, and the diagonal of the causal mask crosses few tiles.
// Four wavefronts of 32 QT rows walk the keys in tiles of 64 that all of them read from LDS.  Scores are formed transposed
// (S^T = K Q^T), so a lane owns one row of the tile; the instruction's rows are assigned to keys (prompt_kperm) so that the eight
// scores of a 16-key step are consecutive keys: they are the B operand of O^T = V^T P^T as they lie.  V^T comes from LDS by transposed reads.
// What bounds it: per 32 keys and 32 rows 4 DP / 32 matrix instructions of 32 clocks, 16 exponentials and ~40 vector instructions;
// an LDS fragment feeds QT matrix instructions, so QT = 2 halves the LDS traffic (QT = 1 needs 128 bytes a clock at full rate).
// Measured: one prompt of 16,384, 32 / 8 heads of 128, QT = 2: 1,890 .. 2,000 us from card to card, 1,930 under the profiler: 1,140 TFLOP/s where an
// 8192^3 product of a library reaches 1,212; 8192 tokens, 32 / 8 heads of 64 265 .. 277 us (QT = 1, with probabilities in two pieces, 486).
// Over the store QT = 1, 8192 tokens, 32 / 8 heads of 128: 915 us.  QT = 2 spills, outside the pipelined loop's steps: 38 registers of a lane
// with heads of 128 (156 bytes of scratch), 15 with heads of 64.
#include "prompt.h"

namespace pserve {

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

__device__ __forceinline__ int prompt_kperm(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

extern __shared__ __attribute__((aligned(16))) uint8_t prompt_smem[];

// Four key rows x 16 values, transposed.  The restricted pointer gives the read an alias scope: without one the compiler takes it
// for a reader of whatever global -> LDS load is in flight and waits for all of them.
__device__ __forceinline__ bf16x4 read_tr16(const lds_u8* __restrict__ p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
}

constexpr int PT_KB = 64;                       // keys of a tile

template <int DP, int QT, int SRC>
struct PromptTileCfg {
    static constexpr int BM = 128 * QT, ROW = DP * 2, TILE = PT_KB * ROW;       // bytes of a key row, of a tile of one operand
    static constexpr int NS = SRC == SRC_STORE ? 2 : 4;
    static constexpr int SCALES = SRC == SRC_STORE ? NS * (2 * PT_KB * 4 + 16) : 0;
    static constexpr int LDS = NS * 2 * TILE + SCALES;
};

// position of 16-byte chunk c of key row r: reads of 16 rows at one chunk (keys) resp. of 4 rows x 64 bytes (values) meet no bank twice
template <int DP> __device__ __forceinline__ int pt_kswz(int r) { return DP == 128 ? r & 15 : (r >> 1) & 7; }
template <int DP> __device__ __forceinline__ int pt_vswz(int r) { return DP == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }

// PAD (packed): heads of fewer than DP values.  Past the head the queries are 0 and another chunk of the key lies in its place; as 0 times
// an infinity is NaN it counts as 0.  Only `half` sees to that: NaN in the pipelined loop sends the block through `half` anyway.
template <int DP, int QT, int SRC, bool PAD>
__global__ void __launch_bounds__(256, QT == 1 || DP == 64 ? 2 : 1)
prompt_tile_kernel(PromptArgs a, int64_t slots) {
    using Cfg = PromptTileCfg<DP, QT, SRC>;
    constexpr bool ST = SRC == SRC_STORE, TWO = ST || QT == 1;
    constexpr int BM = Cfg::BM, ROW = Cfg::ROW, TILE = Cfg::TILE, NS = Cfg::NS;
    constexpr int KS = DP / 16, DT = DP / 32, CP = DP / 8;      // contraction steps, output tiles, chunks of a row
    constexpr int LPO = PT_KB * CP / 256;                       // 16-byte loads a thread and operand

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int fr = lane & 31, fh = lane >> 5;
    const int hk = blockIdx.x % a.Hk, split = (blockIdx.x / a.Hk) % a.splits;
    const int64_t slot = blockIdx.x / (a.Hk * a.splits);
    int s, tile;
    // neighbouring blocks are the key/value heads, so an XCD (block mod 8) stays with few of them and finds their keys in its L2
    if (!prompt_slot<SRC>(a, a.G, BM, slots, slot, s, tile)) return;
    const PromptSeq q = prompt_seq<SRC>(a, s);
    const int64_t rows = (int64_t)q.Lq * a.G, r0 = (int64_t)tile * BM;
    if (tile < 0 || r0 >= rows) return;
    const int nrow = (int)min((int64_t)BM, rows - r0);
    const int ahead = q.Lk - q.Lq;
    auto row_end = [&](int r) { return a.causal ? max(0, min(q.Lk, (int)((r0 + min(r, nrow - 1)) / a.G) + ahead + 1)) : q.Lk; };
    // this block's share of the keys: whole tiles, from `koff` on; keys are numbered from there
    const int all = row_end(nrow - 1);
    const int share = ((all + PT_KB - 1) / PT_KB + a.splits - 1) / a.splits * PT_KB;
    const int koff = (int)min((int64_t)all, (int64_t)split * share);
    const int kend = min(all - koff, share), steps = (kend + PT_KB - 1) / PT_KB;
    auto end_of = [&](int r) { return max(0, min(row_end(r) - koff, kend)); };
    const int w_first = end_of(wave * 32 * QT), w_last = end_of(wave * 32 * QT + 32 * QT - 1);     // keys of the wavefront's first, last row

    // ---- the lane's rows.  A negative scale is taken as that of the negated queries, so that a row's largest score stays its largest
    const u32x4 flip = a.scale2 < 0.f ? u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u} : u32x4{0, 0, 0, 0};
    // (0 is taken as the smallest number, which parts no two scores: a masked one is -infinity, and that times 0 would be NaN)
    const float scale2 = fmaxf(fabsf(a.scale2), 0x1p-149f);
    int tok[QT], head[QT], lim[QT];
    bf16x8 fq[QT][KS];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int r = wave * 32 * QT + 32 * t + fr;
        const int64_t row = r0 + min(r, nrow - 1);
        tok[t] = (int)(row / a.G);
        head[t] = hk * a.G + (int)(row - (int64_t)tok[t] * a.G);
        lim[t] = end_of(r);
        const uint16_t* qp = (const uint16_t*)a.Q + (q.q0 + tok[t]) * a.q_row + (int64_t)head[t] * a.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int d = 16 * ks + 8 * fh;
            const u32x4 w = *reinterpret_cast<const u32x4*>(qp + (d < a.D ? d : 0));
            // past the head: 0
            fq[t][ks] = __builtin_bit_cast(bf16x8, d < a.D ? w ^ flip : u32x4{0, 0, 0, 0});
        }
    }

    // ---- staging
    uint8_t* const sK = prompt_smem;
    uint8_t* const sV = prompt_smem + NS * TILE;
    float* const sS = reinterpret_cast<float*>(prompt_smem + 2 * NS * TILE);    // ST: [NS][64 key scales, 64 value scales]
    uint64_t* const sB = reinterpret_cast<uint64_t*>(prompt_smem + 2 * NS * TILE + NS * 2 * PT_KB * 4);     // ST: [NS] keys that are not there
    // packed: a load of a wavefront fills 64 / CP rows; rows lr + (256 / CP) i
    const int lr = (64 / CP) * wave + lane / CP, lp = lane % CP;
    const int kc = lp ^ pt_kswz<DP>(lr), vc = lp ^ pt_vswz<DP>(lr);             // global chunks of position lp, the same for all i
    const uint8_t* kg = nullptr;
    const uint8_t* vg = nullptr;
    uint32_t k_lane = 0, v_lane = 0;
    if constexpr (!ST) {
        kg = (const uint8_t*)((const uint16_t*)a.K + (q.k0 + koff) * a.k_row + (int64_t)hk * a.k_head);
        vg = (const uint8_t*)((const uint16_t*)a.V + (q.k0 + koff) * a.v_row + (int64_t)hk * a.v_head);
        k_lane = (uint32_t)((lr * (uint32_t)a.k_row + (kc * 8 < a.D ? kc * 8 : 0)) * 2);
        v_lane = (uint32_t)((lr * (uint32_t)a.v_row + (vc * 8 < a.D ? vc * 8 : 0)) * 2);
    }
    // tile min(t, steps - 1) into stage t % NS; rows past the last key repeat it
    auto issue = [&](const uint8_t* base, uint32_t lane_off, int64_t row, uint8_t* ring, int t) {
        const int tt = min(t, steps - 1);
        uint8_t* dst = ring + (t & (NS - 1)) * TILE + wave * 1024;
        const uint8_t* src = base + (int64_t)tt * PT_KB * row * 2;
        const int left = kend - tt * PT_KB;
        if (left >= PT_KB) {
#pragma unroll
            for (int i = 0; i < LPO; ++i)
                __builtin_amdgcn_global_load_lds((const void*)(src + (int64_t)(256 / CP) * i * row * 2 + lane_off), (lds_void*)(dst + i * 4096), 16, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < LPO; ++i) {
                const int r = lr + (256 / CP) * i, up = min(r, left - 1) - lr;
                __builtin_amdgcn_global_load_lds((const void*)(src + ((int64_t)lane_off + (int64_t)up * row * 2)), (lds_void*)(dst + i * 4096), 16, 0, 0);
            }
        }
    };
    auto issue_k = [&](int t) { issue(kg, k_lane, a.k_row, sK, t); };
    auto issue_v = [&](int t) { issue(vg, v_lane, a.v_row, sV, t); };
    // store: 16 whole numbers a load, through registers; rows sr + i * (256 / SC)
    constexpr int SC = DP / 16, SL = PT_KB * SC / 256;          // 16-byte pieces of a row, loads a thread and operand
    const int sr = tid / SC, sc = tid % SC;
    u32x4 rk[ST ? SL : 1], rv[ST ? SL : 1];
    float rs = 0.f;
    bool rbad = false;
    auto place_of = [&](int key) { return prompt_place(a, s, min(key, kend - 1) + koff); };
    int pl[ST ? SL : 1], pls = 0;                               // places of the tile to be fetched next
    auto places = [&](int t) {
#pragma unroll
        for (int i = 0; i < SL; ++i) pl[i] = place_of(t * PT_KB + sr + i * (256 / SC));
        pls = place_of(t * PT_KB + (tid & 63));
    };
    auto fetch = [&]() {
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            const int64_t at = ((int64_t)max(pl[i], 0) * a.Hk + hk) * a.D + (16 * sc < a.D ? 16 * sc : 0);
            rk[i] = *reinterpret_cast<const u32x4*>(a.k8 + at);
            rv[i] = *reinterpret_cast<const u32x4*>(a.v8 + at);
        }
        rs = (tid & 64 ? a.v_scale : a.k_scale)[(int64_t)max(pls, 0) * a.Hk + hk];
        rbad = pls < 0;
    };
    auto put = [&](int st) {
#pragma unroll
        for (int i = 0; i < SL; ++i) {
            const int r = sr + i * (256 / SC);
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const u32x4 w = o ? rv[i] : rk[i];
                uint8_t* row = (o ? sV : sK) + st * TILE + r * ROW;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = (2 * sc + h) ^ (o ? pt_vswz<DP>(r) : pt_kswz<DP>(r));
                    *reinterpret_cast<u32x4*>(row + 16 * c) =
                        u32x4{bf16_of_i8(w[2 * h], 0), bf16_of_i8(w[2 * h], 1), bf16_of_i8(w[2 * h + 1], 0), bf16_of_i8(w[2 * h + 1], 1)};
                }
            }
        }
        if (tid < 128) sS[st * 2 * PT_KB + tid] = rs;
        const uint64_t bad = __ballot(rbad);
        if (tid == 0) sB[st] = bad;
    };

    f32x16 acc[QT][DT];
    float m[QT], l[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = -INFINITY;
        l[t] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[t][d][e] = 0.f;
    }
    const int krow = prompt_kperm(fr);
    // value fragment (half, k2, dt): two transposed reads of four key rows each
    const int vrow = 8 * fh + ((lane & 15) >> 2), vchunk = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vbyte = 8 * (lane & 1);

    // one half (32 keys) of a tile, masked where the wavefront's rows end in it
    auto half = [&](int st, int kv, int H, uint64_t bad) {
        const uint8_t* tk = sK + st * TILE + (krow + 32 * H) * ROW;
        f32x16 sc_[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) sc_[t][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const u32x4 w = *reinterpret_cast<const u32x4*>(tk + 16 * ((2 * ks + fh) ^ pt_kswz<DP>(krow + 32 * H)));
            const bf16x8 fk = __builtin_bit_cast(bf16x8, !PAD || 16 * ks < a.D ? w : u32x4{0, 0, 0, 0});
#pragma unroll
            for (int t = 0; t < QT; ++t) sc_[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk, fq[t][ks], sc_[t], 0, 0, 0);
        }
        const int k0 = kv + 32 * H;
        const uint32_t bad32 = ST ? (uint32_t)(bad >> (32 * H)) : 0u;
        const bool masks = k0 + 32 > w_first || bad32;
        float vs[ST ? 16 : 1];
        if constexpr (ST) {
            const float* ss = sS + st * 2 * PT_KB + 32 * H + 8 * fh;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f32x4 ks_ = *reinterpret_cast<const f32x4*>(ss + 16 * (e >> 3) + (e & 7));
                const f32x4 w = *reinterpret_cast<const f32x4*>(ss + PT_KB + 16 * (e >> 3) + (e & 7));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    vs[e + i] = w[i];
#pragma unroll
                    for (int t = 0; t < QT; ++t) sc_[t][e + i] *= ks_[i];
                }
            }
        }
        uint32_t see[QT];                                       // bit e: the row sees key e of the lane's sixteen
        if (masks) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                see[t] = 0;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = 16 * (e >> 3) + 8 * fh + (e & 7);
                    const bool ok = k0 + j < lim[t] && !(ST && (bad32 >> j & 1));
                    see[t] |= (uint32_t)ok << e;
                    sc_[t][e] = ok ? sc_[t][e] : -INFINITY;
                }
            }
        }
        bf16x8 fp[QT][2], fl[TWO ? QT : 1][2];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            float mx = sc_[t][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sc_[t][e]);
            mx = fmaxf(mx, other_half_f(mx)) * scale2;
            if (__any(mx > m[t])) {
                const float m2 = fmaxf(m[t], mx), f = m2 == m[t] ? 1.f : __builtin_amdgcn_exp2f(m[t] - m2);
                m[t] = m2;
                // (a maximum that overflows only with its scale: the fma below would give finite - infinity, weights of 0, where the row is NaN)
                l[t] = m2 == INFINITY ? __uint_as_float(0x7fc00000u) : l[t] * f;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[t][d][e] *= f;
            }
            const float ref = m[t] == -INFINITY ? 0.f : m[t];
            float p[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                p[e] = __builtin_amdgcn_exp2f(fmaf(sc_[t][e], scale2, -ref));
                l[t] += p[e];
                if constexpr (ST) p[e] = masks && !(see[t] >> e & 1) ? 0.f : p[e] * vs[e];
            }
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2)
                fp[t][k2] = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(p[8 * k2], p[8 * k2 + 1]), pack_bf16x2(p[8 * k2 + 2], p[8 * k2 + 3]),
                                                             pack_bf16x2(p[8 * k2 + 4], p[8 * k2 + 5]), pack_bf16x2(p[8 * k2 + 6], p[8 * k2 + 7])});
            // What the rounding leaves goes along as a second piece, so that the result's own rounding is what is left of the error against 64
            // bits (0.0017 of the norm; with one piece 0.0018 .. 0.0021 for causal prompts, up to 0.0024 where queries see all keys of some
            // thousand at much the same weight).  us with one piece and two, packed: 22 prompts of 77, 12 heads of 64 9.5 and 9.9, 32 of 512 51
            // and 56, 4 of 130 over 4000 keys, 8 / 2 heads of 128 54 and 57.  The tiles of 256 rows, which the matrix cores bound, keep one.
            if constexpr (TWO) {
#pragma unroll
                for (int k2 = 0; k2 < 2; ++k2) {
                    const u32x4 hw = __builtin_bit_cast(u32x4, fp[t][k2]);
                    u32x4 lw;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        lw[e] = pack_bf16x2(p[8 * k2 + 2 * e] - __uint_as_float(hw[e] << 16), p[8 * k2 + 2 * e + 1] - __uint_as_float(hw[e] & 0xffff0000u));
                    fl[t][k2] = __builtin_bit_cast(bf16x8, lw);
                }
            }
        }
#pragma unroll
        for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                bf16x4 h[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int r = 32 * H + 16 * k2 + 4 * u + vrow;
                    h[u] = read_tr16((const lds_u8*)(sV + st * TILE + r * ROW + 16 * ((4 * d + vchunk) ^ pt_vswz<DP>(r)) + vbyte));
                }
                bf16x8 fv = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
                if (!ST && masks) {
                    // a key that a row does not see adds nothing, whatever its value is (0 times a value that is not finite is NaN):
                    // such values count as 0, and a row that sees one gets NaN
                    u32x4 w = __builtin_bit_cast(u32x4, fv), one;
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
                    if (__any(odd)) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t b = ((w[i] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w[i] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                            one[i] = 0x3f803f80u & b;
                            w[i] &= ~b;
                        }
                        fv = __builtin_bit_cast(bf16x8, w);
#pragma unroll
                        for (int t = 0; t < QT; ++t) {
                            u32x4 sees;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t b = see[t] >> (8 * k2 + 2 * i);
                                sees[i] = (b & 1 ? 0x3f80u : 0u) | (b & 2 ? 0x3f800000u : 0u);
                            }
                            f32x16 hit;
#pragma unroll
                            for (int e = 0; e < 16; ++e) hit[e] = 0.f;
                            hit = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, one), __builtin_bit_cast(bf16x8, sees), hit, 0, 0, 0);
#pragma unroll
                            for (int e = 0; e < 16; ++e) acc[t][d][e] = hit[e] > 0.f ? __uint_as_float(0x7fc00000u) : acc[t][d][e];
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    acc[t][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv, fp[t][k2], acc[t][d], 0, 0, 0);
                    if constexpr (TWO) acc[t][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv, fl[t][k2], acc[t][d], 0, 0, 0);
                }
            }
    };

    // The whole tiles of QT = 2, software-pipelined in units of 32 keys x 32 rows: while the exponentials of one unit are formed, the
    // score MFMAs of the next and the output MFMAs of the one before are issued between them (the three do not depend on each other).
    // The softmax reference of a row is the maximum of its first 32 scores and does not move: P = 2^(score - reference) and its sum
    // have the exponent range of fp32, so this is exact unless a later score is 2^60 times larger, or sums overflow with
    // values near the largest number; `wild` then sends the block through the loop with a running maximum.
    bool wild = false;
    auto main_loop = [&](const int whole) {
        f32x16 sa[2];
        u32x4 pk[2][2];                                         // packed probabilities of the unit, 16-key steps
        bf16x8 fk[KS];
        bf16x4 fv[2 * DT][2];                                   // value fragments 16-key step * DT + d
        float nref[2], ls[2] = {0.f, 0.f};
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        // LDS addresses of the fragments, 32 keys further by a constant; they follow the ring tile by tile
        typedef const __attribute__((address_space(3))) u32x4* lds_frag;
        const uint32_t base = (uint32_t)(uintptr_t)(lds_u8*)prompt_smem;
        uint32_t ka[KS], va[DT];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) ka[ks] = base + krow * ROW + 16 * ((2 * ks + fh) ^ pt_kswz<DP>(krow));
#pragma unroll
        for (int d = 0; d < DT; ++d) va[d] = base + NS * TILE + vrow * ROW + 16 * ((4 * d + vchunk) ^ pt_vswz<DP>(vrow)) + vbyte;
        auto read_k = [&](int H, int ks) { fk[ks] = __builtin_bit_cast(bf16x8, *(lds_frag)(uintptr_t)(ka[ks] + 32 * ROW * H)); };
        auto read_v = [&](int H, int j) {
            const int k2 = j / DT, d = j % DT;
#pragma unroll
            for (int u = 0; u < 2; ++u) fv[j][u] = read_tr16((const lds_u8*)(uintptr_t)(va[d] + (32 * H + 16 * k2 + 4 * u) * ROW));
        };
        auto mfma_s = [&](int t, int ks) { sa[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[ks], fq[t][ks], ks == 0 ? zero : sa[t], 0, 0, 0); };
        auto mfma_o = [&](int t, int j) {
            acc[t][j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_shufflevector(fv[j][0], fv[j][1], 0, 1, 2, 3, 4, 5, 6, 7),
                                                                     __builtin_bit_cast(bf16x8, pk[t][j / DT]), acc[t][j % DT], 0, 0, 0);
        };
        // pair g of the unit's sixteen scores
        auto soft = [&](int t, int g) {
            const float e0 = __builtin_amdgcn_exp2f(fmaf(sa[t][2 * g], scale2, nref[t])), e1 = __builtin_amdgcn_exp2f(fmaf(sa[t][2 * g + 1], scale2, nref[t]));
            ls[t] += e0;
            ls[t] += e1;
            pk[t][g / 4][g % 4] = pack_bf16x2(e0, e1);
        };
        constexpr int NJ = KS;                                  // == 2 DT: MFMAs of either kind a unit
        static_assert(KS == 2 * DT, "square units");
        // Nothing that has no side effect stays in its step by itself: what a step forms and what it takes pass through an empty block
        // of assembly at its end.
        auto tie = [&]() {
            asm volatile("" : "+v"(sa[0]), "+v"(sa[1]), "+v"(pk[0][0]), "+v"(pk[0][1]), "+v"(pk[1][0]), "+v"(pk[1][1]), "+v"(ls[0]), "+v"(ls[1]));
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                if constexpr (DP == 128) asm volatile("" : "+a"(acc[0][d]), "+a"(acc[1][d]));
                else asm volatile("" : "+v"(acc[0][d]), "+v"(acc[1][d]));
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        auto order = [&](bool reads) {
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);          // matrix 0x8, LDS read 0x100, transcendental 0x400, other vector 0x2
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (reads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, 8 / NJ, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 24 / NJ, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (reads) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, 8 / NJ, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 24 / NJ, 0);
            }
            tie();
        };
        // unit (H, rows 0): scores of (H, rows 1), outputs of the unit before; fragments are refilled behind their last reader, the keys'
        // with the next half: ka has moved to the next tile when H is 1
        auto step0 = [&](int H) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                mfma_s(1, j);
                read_k(1 - H, j);
                soft(0, (8 * j) / NJ);
                if (NJ == 4) soft(0, 2 * j + 1);
                mfma_o(1, j);
                read_v(H, j);
            }
            order(true);
        };
        auto step1 = [&]() {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                mfma_s(0, j);
                soft(1, (8 * j) / NJ);
                if (NJ == 4) soft(1, 2 * j + 1);
                mfma_o(0, j);
            }
            order(false);
        };
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(4 * LPO) : "memory");     // K tile 0
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) read_k(0, ks);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) mfma_s(t, ks);
            float mx = sa[t][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) mx = fmaxf(mx, sa[t][e]);
            mx = fmaxf(mx, other_half_f(mx)) * scale2;
            m[t] = mx;
            nref[t] = -mx;
            pk[t][0] = pk[t][1] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int j = 0; j < 2 * DT; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) fv[j][u] = __builtin_bit_cast(bf16x4, q8_u32x2{0, 0});     // the first outputs add 0 * 0
        // DP = 128: the accumulators and the queries live in the second half of the register file, which leaves the first to what the
        // vector unit touches; DP = 64: two blocks a CU, and no second half
        if constexpr (DP == 128) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+a"(fq[t][ks]));
        }
        tie();
        for (int t = 0; t < whole; ++t) {
            asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * LPO) : "memory");
            const uint32_t next = (t & (NS - 1)) == NS - 1 ? (uint32_t)-((NS - 1) * TILE) : (uint32_t)TILE;
            step0(0);
            issue_k(t + 3);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) ka[ks] += next;
            tie();
            step1();
            issue_v(t + 2);
            tie();
            step0(1);
            step1();
#pragma unroll
            for (int d = 0; d < DT; ++d) va[d] += next;
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) mfma_o(1, j);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            l[t] = ls[t];
            wild |= !(ls[t] < 0x1p60f) || m[t] == INFINITY;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) wild |= !(fabsf(acc[t][d][e]) < 0x1p126f);
        }
    };

    if (steps > 0) {
        if constexpr (ST) {
            places(0);
            fetch();
            places(1);
            for (int t = 0; t < steps; ++t) {
                put(t & 1);
                if (t + 1 < steps) {
                    fetch();
                    places(t + 2);
                }
                __syncthreads();
                const uint64_t bad = sB[t & 1];
                const int kv = t * PT_KB;
                if (kv < w_last) {
                    half(t & 1, kv, 0, bad);
                    if (kv + 32 < w_last) half(t & 1, kv, 1, bad);
                }
            }
        } else {
            int whole = 0;                                      // tiles that all rows of the block see whole
            if constexpr (QT == 2) whole = end_of(0) / PT_KB;
            for (;;) {
                issue_k(0);
                issue_k(1);
                issue_v(0);
                issue_k(2);
                issue_v(1);
                int t = 0;
                if constexpr (QT == 2) {
                    if (whole > 0) {
                        main_loop(whole);
                        t = whole;
                    }
                }
                for (; t < steps; ++t) {
                    // K of tile t + 1 and V of tile t have landed, and every wavefront is through with the tiles whose stages are loaded
                    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * LPO) : "memory");
                    issue_k(t + 3);
                    issue_v(t + 2);
                    const int kv = t * PT_KB;
                    if (kv < w_last) {
                        half(t & (NS - 1), kv, 0, 0);
                        if (kv + 32 < w_last) half(t & (NS - 1), kv, 1, 0);
                    }
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // no load may still write LDS when the block ends or starts over
                if (whole == 0) break;
                // Did the main loop stay in range?  Else everything again, in the loop with a running maximum
                __syncthreads();
                uint32_t* vote = reinterpret_cast<uint32_t*>(prompt_smem);
                if (lane == 0) vote[wave] = 0;
                if (__any(wild) && lane == 0) vote[wave] = 1;
                __syncthreads();
                const bool again = (vote[0] | vote[1] | vote[2] | vote[3]) != 0;
                __syncthreads();
                if (!again) break;
                whole = 0;
#pragma unroll
                for (int i = 0; i < QT; ++i) {
                    m[i] = -INFINITY;
                    l[i] = 0.f;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[i][d][e] = 0.f;
                }
            }
        }
    }

    if (a.splits > 1) {                                         // [row][DP] accumulators, [row] references, [row] sums
        float* part = a.part + ((slot * a.splits + split) * a.Hk + hk) * (int64_t)(BM * (DP + 2));
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float ll = l[t] + other_half_f(l[t]);
            const int r = wave * 32 * QT + 32 * t + fr;
            if (r >= nrow) continue;
            if (fh == 0) { part[BM * DP + r] = m[t]; part[BM * DP + BM + r] = ll; }
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int eg = 0; eg < 4; ++eg)
                    *reinterpret_cast<f32x4*>(part + r * DP + 32 * d + 8 * eg + 4 * fh) =
                        f32x4{acc[t][d][4 * eg], acc[t][d][4 * eg + 1], acc[t][d][4 * eg + 2], acc[t][d][4 * eg + 3]};
        }
        return;
    }
    // ---- O[row][d] = O^T / l; the lane has d = 32 dt + 8 (e / 4) + 4 fh + e % 4 of its rows, lane ^ 32 the next four: they trade
    // so that one has the even groups of eight and the other the odd ones
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const float ll = l[t] + other_half_f(l[t]);
        const float inv = ll == 0.f ? 0.f : 1.f / ll;           // a row without keys: 0
        if (wave * 32 * QT + 32 * t + fr >= nrow) continue;     // (both lanes of a row together)
        uint16_t* op = (uint16_t*)a.O + (q.q0 + tok[t]) * a.o_row + (int64_t)head[t] * a.o_head + 8 * fh;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int eg = 0; eg < 4; eg += 2) {
                uint32_t w[2][2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    w[i][0] = pack_bf16x2(acc[t][d][4 * (eg + i)] * inv, acc[t][d][4 * (eg + i) + 1] * inv);
                    w[i][1] = pack_bf16x2(acc[t][d][4 * (eg + i) + 2] * inv, acc[t][d][4 * (eg + i) + 3] * inv);
                }
                const auto x0 = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
                const auto x1 = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                if (32 * d + 8 * eg + 8 * fh < a.D) *reinterpret_cast<u32x4*>(op + 32 * d + 8 * eg) = u32x4{x0[0], x1[0], x0[1], x1[1]};
            }
    }
}

template <int DP, int QT, int SRC, bool PAD = false>
static int launch_tile_as(const PromptArgs& a, hipStream_t st) {
    using Cfg = PromptTileCfg<DP, QT, SRC>;
    PS_SET_LDS_ONCE((prompt_tile_kernel<DP, QT, SRC, PAD>), Cfg::LDS);
    const int64_t slots = prompt_slots(a, a.G, Cfg::BM);
    prompt_tile_kernel<DP, QT, SRC, PAD><<<(unsigned)(slots * a.Hk * a.splits), 256, Cfg::LDS, st>>>(a, slots);
    PS_TRY(check_launch("prompt_tile_kernel"));
    return a.splits > 1 ? launch_prompt_join(a, SRC, st) : PSERVE_OK;
}

int launch_prompt_tile(const PromptArgs& a, int rows, int src, hipStream_t st) {
    if (src == SRC_STORE) return a.D <= 64 ? launch_tile_as<64, 1, SRC_STORE>(a, st) : launch_tile_as<128, 1, SRC_STORE>(a, st);
    if (a.D < 64) return rows == 128 ? launch_tile_as<64, 1, SRC_PACKED, true>(a, st) : launch_tile_as<64, 2, SRC_PACKED, true>(a, st);
    if (a.D == 64) return rows == 128 ? launch_tile_as<64, 1, SRC_PACKED>(a, st) : launch_tile_as<64, 2, SRC_PACKED>(a, st);
    if (a.D < 128) return rows == 128 ? launch_tile_as<128, 1, SRC_PACKED, true>(a, st) : launch_tile_as<128, 2, SRC_PACKED, true>(a, st);
    return rows == 128 ? launch_tile_as<128, 1, SRC_PACKED>(a, st) : launch_tile_as<128, 2, SRC_PACKED>(a, st);
}

}  // namespace pserve
