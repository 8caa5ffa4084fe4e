// Causal attention with grouped heads, gfx950: tiles of 16 rows, keys shared out between wavefronts and blocks.
//
// A row is a query token's head; the G heads that share a key/value head are neighbouring rows of that head's tile, so one pass
// over keys and values serves them all.  A block's four wavefronts take 32 keys (fp32: 16) of a tile at a time in turn, each with a
// softmax of its own (running maximum and sum in fp32), and meet in LDS at the end.  Where there are tiles enough a block has whole
// ones; where there are few, or few with many keys, all tiles' keys are cut into units of 128, the blocks take equal runs of
// them whatever the sequences' lengths are, and a second kernel joins the tiles that more than one block has.
//
// Scores are formed transposed, S^T = K Q^T on 16 x 16 matrix instructions, so a lane owns one row and NV consecutive keys; the keys
// of a step are assigned to the instruction's rows so that the lane's probabilities are the B operand of O^T = V^T P^T as they lie.
// bf16: V passes LDS row by row and is read back transposed (ds_read_b64_tr); fp32: V comes from memory in the operand's layout.
// Keys and values in 8 bits are exact as bf16 numbers; the scale of a key multiplies its score, that of a value its probability.
// What bounds it: over the store the bytes of keys and values, G rows at a time (one token over 131,072 keys, 32 / 8 heads of 128: 55 us, 5.0
// of the 5.15 TB/s of a copy, and 10 to join; 32 tokens over 12 .. 8000 keys 31 and 7); packed fp32 the matrix instructions.
#include "prompt.h"

namespace pserve {

typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef float __attribute__((ext_vector_type(4), aligned(4))) f32x4_4;          // of four bytes' alignment
typedef __attribute__((address_space(3))) q8_u32x2 lds_u32x2;
typedef __attribute__((ext_vector_type(2))) int i32x2;
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

constexpr float NEG_INF = -INFINITY;

// bytes of one wavefront's value tile in LDS: 32 rows
template <typename T, int DP, int SRC> constexpr int few_v_bytes() { return sizeof(T) == 4 ? 0 : 32 * DP * (SRC == SRC_STORE ? 1 : 2); }

// DV consecutive values of a row, times inv
template <int DV, typename T>
__device__ __forceinline__ void store_row(T* p, const float (&o)[DV], float inv) {
    if constexpr (sizeof(T) == 2) {
        uint32_t w[DV / 2];
#pragma unroll
        for (int i = 0; i < DV / 2; ++i) w[i] = pack_bf16x2(o[2 * i] * inv, o[2 * i + 1] * inv);
        if constexpr (DV == 8) *reinterpret_cast<u32x4*>(p) = u32x4{w[0], w[1], w[2], w[3]};
        else *reinterpret_cast<q8_u32x2*>(p) = q8_u32x2{w[0], w[1]};
    } else {
#pragma unroll
        for (int i = 0; i < DV; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv};
    }
}

// DP: the head's values, rounded up to 64 or 128.  DX: sixteenths of a head that are computed.  Packed fp32 heads, which the matrix
// instructions bound (4096 tokens, 2 x 4 heads of 128: 370 us, 93 of the 154 TFLOP/s of a large product), have D / 16: heads of 80 take 255 us,
// filled up to 128 they took what those do.  Elsewhere DP / 16.
// PAD (packed bf16): D < DP.  What is read in place of a key's values past the head counts as 0: the queries are 0 there, but 0 times an
// infinity is NaN.
template <typename T, int DP, int SRC, int DX, bool PAD>
__global__ void __launch_bounds__(256, 2)
prompt_few_kernel(PromptArgs a) {
    constexpr bool F32 = sizeof(T) == 4, ST = SRC == SRC_STORE, EXACT = F32 && !ST;
    constexpr int KT = F32 ? 16 : 32, NV = KT / 4, DT = DX;
    constexpr int KS = F32 ? 4 * DX : DP / 32;              // contraction steps of a score
    constexpr int NQ = KS;
    constexpr int BUF_ROW = DP + 4;                         // floats of a row in the meeting place (16 bytes of padding: banks)
    constexpr int VB = few_v_bytes<T, DP, SRC>();
    constexpr int MEET = 4 * 16 * BUF_ROW * 4, SMEM = MEET > 4 * VB ? MEET : 4 * VB;
    __shared__ __attribute__((aligned(16))) uint8_t smem[SMEM];
    __shared__ float s_ml[4][16][2];
    __shared__ __attribute__((aligned(16))) float s_scale[ST ? 4 : 1][64];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g4 = lane >> 4;
    const int64_t b = blockIdx.x;
    PromptWalk<SRC> walk(a);
    int64_t w = b, w_lo = 0, w_end = a.items;
    if (a.unit) {
        const int64_t W = walk.total();
        if (b >= W) return;
        const PromptShares shares(a, W);
        w = w_lo = shares.begin(b);
        w_end = shares.begin(b + 1);
    }
    for (bool again = false; w < w_end; again = true) {
    if (again) __syncthreads();                             // LDS is taken again
    PromptSeq q;
    int s, tile, hk, off = 0, take = 1, U = 1;
    bool first = true;
    if (a.unit) {
        // ---- the next run of units: a tile's, or what the block has of it
        if (!walk.find(w)) return;
        q = walk.seq();
        s = walk.s;
        U = walk.tile_units();
        const int item = prompt_item(w - walk.base, U, off);
        tile = item / a.Hk;
        hk = item - tile * a.Hk;
        take = (int)min((int64_t)(U - off), w_end - w);
        first = w == w_lo;
        w += take;
    } else {
        // ---- a whole tile
        const uint32_t item = (uint32_t)w, slot = item / (uint32_t)a.Hk;
        w += gridDim.x;
        hk = (int)(item - slot * (uint32_t)a.Hk);
        if (!prompt_slot<SRC>(a, a.G, 16, a.items / a.Hk, slot, s, tile)) continue;
        tile = __builtin_amdgcn_readfirstlane(tile);
        q = prompt_seq<SRC>(a, s);
        q.q0 = uniform64(q.q0);
        q.k0 = uniform64(q.k0);
        q.Lq = __builtin_amdgcn_readfirstlane(q.Lq);
        q.Lk = __builtin_amdgcn_readfirstlane(q.Lk);
        if (tile < 0 || (int64_t)tile * 16 >= (int64_t)q.Lq * a.G) continue;
    }
    const int64_t rows = (int64_t)q.Lq * a.G, r0 = (int64_t)tile * 16;
    const int nrow = (int)min((int64_t)16, rows - r0);

    // the lane's row, and the end of the keys it sees
    const int64_t row = r0 + min(col, nrow - 1);
    const int tok = (int)(row / a.G), head = hk * a.G + (int)(row - (int64_t)tok * a.G);
    const int ahead = q.Lk - q.Lq;                          // queries stand at the end of the keys
    const int row_end = a.causal ? max(0, min(q.Lk, tok + ahead + 1)) : q.Lk;
    const int tok_last = (int)((r0 + nrow - 1) / a.G);
    const int all = a.causal ? max(0, min(q.Lk, tok_last + ahead + 1)) : q.Lk;      // keys of the tile
    const int kbeg = (int)min((int64_t)all, (int64_t)max(0, off - a.lead) * a.unit);
    const int kend = a.unit ? (int)min((int64_t)all, (int64_t)max(0, off + take - a.lead) * a.unit) : all;
    const int lim = min(row_end, kend);                     // the row's keys are those below

    // ---- query fragments, in the order of the contraction that the key loads below give
    bf16x8 qb[F32 ? 1 : NQ];
    float qf[F32 ? NQ : 1];
    {
        const T* qp = (const T*)a.Q + (q.q0 + tok) * a.q_row + (int64_t)head * a.q_head;
#pragma unroll
        for (int i = 0; i < (F32 ? NQ / 4 : NQ); ++i) {
            // first value of the lane's i-th chunk of 8 (fp32: 4) values
            const int d = F32 ? (ST ? 64 * (i / 4) + 16 * g4 + 4 * (i % 4) : 16 * i + 4 * g4)
                              : (ST ? 64 * (i / 2) + 16 * g4 + 8 * (i % 2) : 32 * i + 8 * g4);
            const bool in = d < a.D;                        // D is a multiple of 16: a chunk is inside or outside
            const u32x4 w = *reinterpret_cast<const u32x4*>(qp + (in ? d : 0));
            if constexpr (F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) qf[4 * i + e] = in ? __uint_as_float(w[e]) : 0.f;
            } else {
                qb[i] = __builtin_bit_cast(bf16x8, in ? w : u32x4{0, 0, 0, 0});
            }
        }
    }

    // ---- what a wavefront holds of a step: keys in fragment order, values by rows (bf16) or in operand order (fp32)
    constexpr int NK = F32 ? (ST ? DP / 64 : DX) : 2 * (ST ? DP / 64 : DP / 32);
    constexpr int NVL = F32 ? (ST ? 4 : 1) : (ST ? DP / 32 : DP / 16);
    struct Step {
        u32x4 k[NK], v[NVL];
        float vf[EXACT ? 4 : 1][DX];
        float scale;
        uint32_t bad;                                       // keys whose place is none of the store's
    };
    const T* kb_ = ST ? nullptr : (const T*)a.K + q.k0 * a.k_row + (int64_t)hk * a.k_head;
    const T* vb_ = ST ? nullptr : (const T*)a.V + q.k0 * a.v_row + (int64_t)hk * a.v_head;
    // store: the place of key (kb + lane % KT), -1: none
    auto place_of = [&](int kb) {
        return prompt_place(a, s, min(kb + (lane & (KT - 1)), kend - 1));
    };
    auto load = [&](Step& f, int kb, int place) {
        auto key_at = [&](int j) { return min(kb + j, kend - 1); };
        const int pl = ST ? max(place, 0) : 0;
        if constexpr (ST) {
            f.bad = (uint32_t)__ballot(place < 0) & (KT == 32 ? 0xffffffffu : 0xffffu);
            const bool vs = F32 ? (lane & 16) != 0 : lane >= 32;
            f.scale = (vs ? a.v_scale : a.k_scale)[(int64_t)pl * a.Hk + hk];
        }
        // keys
        if constexpr (ST) {
#pragma unroll
            for (int t = 0; t < (F32 ? 1 : 2); ++t) {
                const int j = F32 ? col : 8 * (col >> 2) + 4 * t + (col & 3);
                const int8_t* p = a.k8 + ((int64_t)__shfl(pl, j) * a.Hk + hk) * a.D;
#pragma unroll
                for (int i = 0; i < DP / 64; ++i) {
                    const int d = 64 * i + 16 * g4;
                    f.k[t * (DP / 64) + i] = *reinterpret_cast<const u32x4*>(p + (d < a.D ? d : 0));
                }
            }
        } else {
#pragma unroll
            for (int t = 0; t < (F32 ? 1 : 2); ++t) {
                const int j = F32 ? col : 8 * (col >> 2) + 4 * t + (col & 3);
                const T* p = kb_ + (int64_t)key_at(j) * a.k_row;
                constexpr int CH = F32 ? 4 : 8, NC = F32 ? DX : DP / 32;
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const int d = 4 * CH * i + CH * g4;
                    f.k[t * NC + i] = *reinterpret_cast<const u32x4*>(p + (d < a.D ? d : 0));
                }
            }
        }
        // values
        if constexpr (F32 && ST) {
            // the lane's DP / 16 values of each of its four keys
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = min(col * (DP / 16), a.D - DP / 16);
                const int8_t* p = a.v8 + ((int64_t)__shfl(pl, 4 * g4 + i) * a.Hk + hk) * a.D + d;
                if constexpr (DP == 128) {
                    const q8_u32x2 w = *reinterpret_cast<const q8_u32x2*>(p);
                    f.v[i][0] = w[0]; f.v[i][1] = w[1];
                } else {
                    f.v[i][0] = *reinterpret_cast<const uint32_t*>(p);
                }
            }
        } else if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const T* p = vb_ + (int64_t)key_at(4 * g4 + i) * a.v_row;
                p += col * DX;
                if constexpr (DX >= 4) {
                    f32x4 w;
                    if constexpr (DX % 4 == 0) w = *reinterpret_cast<const f32x4*>(p);
                    else w = *reinterpret_cast<const f32x4_4*>(p);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f.vf[i][e] = w[e];
                }
                if constexpr (DX == 8) {
                    const f32x4 w = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f.vf[i][4 + e] = w[e];
                } else {
#pragma unroll
                    for (int e = DX / 4 * 4; e < DX; ++e) f.vf[i][e] = p[e];
                }
            }
        } else {
            constexpr int CH = ST ? 16 : 8, CP = DP / CH;   // values of a 16-byte chunk, chunks of a row
#pragma unroll
            for (int i = 0; i < NVL; ++i) {
                const int idx = 64 * i + lane, j = idx / CP, c = idx % CP, d = c * CH < a.D ? c * CH : 0;
                if constexpr (ST) f.v[i] = *reinterpret_cast<const u32x4*>(a.v8 + ((int64_t)__shfl(pl, j) * a.Hk + hk) * a.D + d);
                else f.v[i] = *reinterpret_cast<const u32x4*>(vb_ + (int64_t)key_at(j) * a.v_row + d);
            }
        }
    };

    f32x4 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = NEG_INF, l = 0.f;
    uint8_t* sv = smem + wave * VB;

    // row positions of the value tile in LDS: 16-byte chunk c of row j lies at chunk c ^ swz(j), so that the 16 rows that a
    // transposed read touches at a time lie in different banks
    auto swz = [](int j) -> int {
        if constexpr (ST) return DP == 128 ? (j >> 1) & 7 : (j >> 2) & 3;
        else return DP == 128 ? ((j & 3) << 1) | (((j >> 3) & 1) << 3) : (((j >> 1) & 1) << 1) | (((j >> 3) & 1) << 2);
    };

    auto step = [&](const Step& f, int kb) {
        int ln = lane;
        asm volatile("" : "+v"(ln));                        // LDS addresses are formed here, not ahead of the loop (registers)
        const int col = ln & 15, g4 = ln >> 4;
        // ---- scores of the lane's row and its NV keys kb + NV g4 ..
        float x[NV];
        if constexpr (F32) {
            f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                float kv;
                if constexpr (ST) kv = (float)(int8_t)(f.k[i / 16][(i / 4) % 4] >> (8 * (i % 4)));
                else kv = __uint_as_float(f.k[i / 4][i % 4]);
                sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kv, qf[i], sc, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = sc[e];
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    bf16x8 fk;
                    if constexpr (ST) {
                        const u32x4 w = f.k[t * (DP / 64) + i / 2];
                        const uint32_t w0 = w[2 * (i % 2)], w1 = w[2 * (i % 2) + 1];
                        fk = __builtin_bit_cast(bf16x8, u32x4{bf16_of_i8(w0, 0), bf16_of_i8(w0, 1), bf16_of_i8(w1, 0), bf16_of_i8(w1, 1)});
                    } else {
                        const u32x4 w = f.k[t * (DP / 32) + i];
                        fk = __builtin_bit_cast(bf16x8, !PAD || 32 * i + 8 * g4 < a.D ? w : u32x4{0, 0, 0, 0});
                    }
                    sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fk, qb[i], sc, 0, 0, 0);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * t + e] = sc[e];
            }
        }
        float vs[NV];
        if constexpr (ST) {
            s_scale[wave][ln] = f.scale;
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int j = 0; j < NV; j += 4) {
                const f32x4 ks = *reinterpret_cast<const f32x4*>(&s_scale[wave][NV * g4 + j]);
                const f32x4 w = *reinterpret_cast<const f32x4*>(&s_scale[wave][KT + NV * g4 + j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) { x[j + e] = x[j + e] * ks[e] * a.scale2; vs[j + e] = w[e]; }    // (the scales' product may overflow)
            }
            __builtin_amdgcn_wave_barrier();
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) x[j] *= a.scale2;
        }
        const bool masks = __any(kb + KT > lim) || (ST && f.bad);
        bool ok[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) ok[j] = true;
        if (masks) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                ok[j] = kb + NV * g4 + j < lim && !(ST && (f.bad >> (NV * g4 + j) & 1));
                x[j] = ok[j] ? x[j] : NEG_INF;
            }
        }
        // ---- softmax: reference = running maximum of the row (log2 domain)
        float mx = x[0];
#pragma unroll
        for (int j = 1; j < NV; ++j) mx = fmaxf(mx, x[j]);
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        if (__any(mx > m)) {
            const float m2 = fmaxf(m, mx), f_ = m2 == m ? 1.f : __builtin_amdgcn_exp2f(m - m2);
            m = m2;
            l *= f_;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[t][e] *= f_;
        }
        const float ref = m == NEG_INF ? 0.f : m;
        float p[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            p[j] = __builtin_amdgcn_exp2f(x[j] - ref);
            l += p[j];
            if constexpr (ST) p[j] = masks && !ok[j] ? 0.f : p[j] * vs[j];
        }
        // ---- O^T += V^T P^T.  A masked key adds nothing, whatever its value is: 0 times a value that is not finite would be NaN
        if constexpr (F32) {
            float vv[4][DT];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    if constexpr (ST) vv[i][t] = (float)(int8_t)(f.v[i][t / 4] >> (8 * (t % 4)));
                    else vv[i][t] = f.vf[i][t];
                }
            if (!ST && masks) {
                bool odd = false;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int t = 0; t < DT; ++t) odd |= abs_bits(vv[i][t]) >= 0x7f800000u;
                if (__any(odd)) {
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        f32x4 hit = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bool o = abs_bits(vv[i][t]) >= 0x7f800000u;
                            hit = __builtin_amdgcn_mfma_f32_16x16x4f32(o ? 1.f : 0.f, ok[i] ? 1.f : 0.f, hit, 0, 0, 0);
                            vv[i][t] = o ? 0.f : vv[i][t];
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t][e] = hit[e] > 0.f ? __uint_as_float(0x7fc00000u) : acc[t][e];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < DT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[i][t], p[i], acc[t], 0, 0, 0);
        } else {
            const bf16x8 fp = __builtin_bit_cast(bf16x8, u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4 % NV], p[5 % NV]),
                                                               pack_bf16x2(p[6 % NV], p[7 % NV])});
            // what the rounding to bf16 leaves of a probability (up to 2^-8 of it, as much as the output's own rounding) goes through the
            // matrix cores as a second piece; of that up to 2^-8 is lost in turn
            const u32x4 hw = __builtin_bit_cast(u32x4, fp);
            u32x4 lw;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                lw[e] = pack_bf16x2(p[(2 * e) % NV] - __uint_as_float(hw[e] << 16), p[(2 * e + 1) % NV] - __uint_as_float(hw[e] & 0xffff0000u));
            const bf16x8 fl = __builtin_bit_cast(bf16x8, lw);
            constexpr int CP = DP / (ST ? 16 : 8), RB = DP * (ST ? 1 : 2);      // chunks, bytes of a row
            bool odd = false;
#pragma unroll
            for (int i = 0; i < NVL; ++i) {
                const int idx = 64 * i + ln, j = idx / CP, c = idx % CP;
                *reinterpret_cast<u32x4*>(sv + j * RB + ((c ^ swz(j)) << 4)) = f.v[i];
                if (!ST && masks) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd |= (f.v[i][e] & 0x7f80u) == 0x7f80u || (f.v[i][e] & 0x7f800000u) == 0x7f800000u;
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            odd = !ST && masks && __any(odd);
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                bf16x8 fv;
                if constexpr (ST) {
                    const int j = 8 * g4 + (col >> 1);
                    const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(lds_u8*)(sv + j * RB + ((t ^ swz(j)) << 4) + 8 * (col & 1)));
                    const uint32_t w0 = (uint32_t)w[0], w1 = (uint32_t)w[1];
                    fv = __builtin_bit_cast(bf16x8, u32x4{bf16_of_i8(w0, 0), bf16_of_i8(w0, 1), bf16_of_i8(w1, 0), bf16_of_i8(w1, 1)});
                } else {
                    bf16x4 h[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int j = 8 * g4 + 4 * u + (col >> 2), c = 2 * t + ((col & 3) >> 1);
                        h[u] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(lds_u8*)(sv + j * RB + ((c ^ swz(j)) << 4) + 8 * (col & 1)));
                    }
                    fv = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    if (odd) {
                        u32x4 w = __builtin_bit_cast(u32x4, fv), bad;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t lo = (w[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
                            bad[e] = 0x3f803f80u & (lo | hi);
                            w[e] &= ~(lo | hi);
                        }
                        u32x4 see;
#pragma unroll
                        for (int e = 0; e < 4; ++e) see[e] = (ok[(2 * e) % NV] ? 0x3f80u : 0u) | (ok[(2 * e + 1) % NV] ? 0x3f800000u : 0u);
                        f32x4 hit = {0.f, 0.f, 0.f, 0.f};
                        hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, bad), __builtin_bit_cast(bf16x8, see), hit, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[t][e] = hit[e] > 0.f ? __uint_as_float(0x7fc00000u) : acc[t][e];
                        fv = __builtin_bit_cast(bf16x8, w);
                    }
                }
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv, fp, acc[t], 0, 0, 0);
                acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv, fl, acc[t], 0, 0, 0);
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();                // the next step's rows come after these reads
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    };

    // ---- the wavefront's steps, one ahead in registers (behind the last one the last keys again; two ahead took 42 us where one takes 38,
    // 32 sequences of 12 .. 8000 tokens).  Loads come back in order, so the table entries of a step are asked for in front of the keys and
    // values of the step before it
    constexpr int KS4 = 4 * KT;
    int kb = kbeg + wave * KT;
    if (kb < kend) {
        Step cur, nxt;
        int place = 0, after = 0;
        if constexpr (ST) {
            place = place_of(kb);
            after = place_of(kb + KS4);
        }
        load(cur, kb, place);
#pragma unroll 1
        for (; kb < kend; kb += KS4) {
            place = after;
            if constexpr (ST) after = place_of(kb + 2 * KS4);
            load(nxt, kb + KS4, place);
            step(cur, kb);
            cur = nxt;
        }
    }

    // ---- the four wavefronts meet
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    __syncthreads();                                        // value tiles are done with
    float* buf = reinterpret_cast<float*>(smem);
    if (g4 == 0) { s_ml[wave][col][0] = m; s_ml[wave][col][1] = l; }
    {
        float* to = buf + (wave * 16 + col) * BUF_ROW;
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            if constexpr (F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) to[(4 * g4 + e) * DX + t] = acc[t][e];
            } else {
                *reinterpret_cast<f32x4*>(to + 16 * t + 4 * g4) = acc[t];
            }
        }
    }
    __syncthreads();
    const int r = tid >> 4, d0 = (tid & 15) * (DP / 16);
    if (r >= nrow) continue;
    float mm = NEG_INF, ll = 0.f, o[DP / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i) mm = fmaxf(mm, s_ml[i][r][0]);
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) o[i] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float mw = s_ml[i][r][0], f = mw == mm ? 1.f : __builtin_amdgcn_exp2f(mw - mm);
        ll += s_ml[i][r][1] * f;
#pragma unroll
        for (int e = 0; e < DP / 16; ++e) o[e] += buf[(i * 16 + r) * BUF_ROW + d0 + e] * f;
    }
    if (take < U) {
        float* part = a.part + (2 * b + !first) * (16 * (DP + 2));
        if ((tid & 15) == 0) { part[16 * DP + r] = mm; part[16 * DP + 16 + r] = ll; }
#pragma unroll
        for (int e = 0; e < DP / 16; e += 4) *reinterpret_cast<f32x4*>(part + r * DP + d0 + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
        continue;
    }
    if (d0 >= a.D) continue;
    const int64_t rr = r0 + r;
    const int tk = (int)(rr / a.G), hd = hk * a.G + (int)(rr - (int64_t)tk * a.G);
    T* op = (T*)a.O + (q.q0 + tk) * a.o_row + (int64_t)hd * a.o_head + d0;
    store_row<DP / 16>(op, o, ll == 0.f ? 0.f : 1.f / ll);  // a row without keys: 0
    }
}

// Joins the runs of the tiles that more than one block has.  Such a tile holds the first unit of a block: block b takes the tile that
// holds its own first unit, unless the one before it does already.  16 threads a row; few rows share out the runs between them.
template <typename T, int DP, int SRC>
__global__ void __launch_bounds__(512)
prompt_meet_kernel(PromptArgs a) {
    constexpr int DV = DP / 16, SLOTS = 32, RU = 4;         // rows x groups of runs of a block, runs in flight
    __shared__ float s_o[SLOTS][DP], s_ml[SLOTS][2];
    PromptWalk<SRC> walk(a);
    const PromptShares shares(a, walk.total());
    const int64_t b0 = blockIdx.x;                          // the first block that has the tile
    if (b0 + 1 >= shares.B) return;
    const int64_t lo = shares.begin(b0), w = shares.begin(b0 + 1);
    if (!walk.find(w)) return;
    const int U = walk.tile_units();
    int off;
    const int item = prompt_item(w - walk.base, U, off), tile = item / a.Hk, hk = item - tile * a.Hk;
    const int64_t w0 = w - off, w1 = w0 + U;
    if (off == 0 || (b0 > 0 && lo > w0)) return;            // no tile is cut here, or it is cut further in front, too
    const PromptSeq q = walk.seq();
    const int runs = (int)(shares.block_of(w1 - 1) - b0) + 1;
    const int64_t rows = (int64_t)q.Lq * a.G, r0 = (int64_t)tile * 16;
    const int nrow = (int)min((int64_t)16, rows - r0), per = nrow <= 2 ? 2 : nrow <= 4 ? 4 : nrow <= 8 ? 8 : 16, groups = SLOTS / per;
    const int part_row = threadIdx.x >> 4, r = part_row % per, group = part_row / per, d0 = (threadIdx.x & 15) * DV;
    // a block's run of this tile is its first one (2 b), but for a first block that begins with another tile
    const int late = lo < w0 ? 1 : 0;
    auto part_of = [&](int i) { return a.part + (2 * (b0 + i) + (i == 0 ? late : 0)) * (16 * (DP + 2)); };
    float mm = NEG_INF, ll = 0.f, o[DV];
#pragma unroll
    for (int e = 0; e < DV; ++e) o[e] = 0.f;
    if (r < nrow) {
        for (int i = group; i < runs; i += RU * groups) {   // (references, sums and values of RU runs in one go)
            float mw[RU], lw[RU];
            f32x4 v[RU][DV / 4];
#pragma unroll
            for (int u = 0; u < RU; ++u) {
                const float* p = part_of(min(i + u * groups, runs - 1));
                mw[u] = p[16 * DP + r];
                lw[u] = p[16 * DP + 16 + r];
#pragma unroll
                for (int e = 0; e < DV / 4; ++e) v[u][e] = *reinterpret_cast<const f32x4*>(p + r * DP + d0 + 4 * e);
            }
            float m2 = mm;
#pragma unroll
            for (int u = 0; u < RU; ++u) m2 = fmaxf(m2, mw[u]);
            const float f0 = mm == m2 ? 1.f : __builtin_amdgcn_exp2f(mm - m2);
            mm = m2;
            ll *= f0;
#pragma unroll
            for (int e = 0; e < DV; ++e) o[e] *= f0;
#pragma unroll
            for (int u = 0; u < RU; ++u) {
                if (i + u * groups >= runs) break;
                const float f = mw[u] == mm ? 1.f : __builtin_amdgcn_exp2f(mw[u] - mm);
                ll += lw[u] * f;
#pragma unroll
                for (int e = 0; e < DV; ++e) o[e] += v[u][e / 4][e % 4] * f;
            }
        }
    }
    if ((threadIdx.x & 15) == 0) { s_ml[part_row][0] = mm; s_ml[part_row][1] = ll; }
#pragma unroll
    for (int e = 0; e < DV; ++e) s_o[part_row][d0 + e] = o[e];
    __syncthreads();
    if (group || r >= nrow || d0 >= a.D) return;
    for (int i = 1; i < groups; ++i) mm = fmaxf(mm, s_ml[i * per + r][0]);
    ll = 0.f;
#pragma unroll
    for (int e = 0; e < DV; ++e) o[e] = 0.f;
    for (int i = 0; i < groups; ++i) {
        const float mw = s_ml[i * per + r][0], f = mw == mm ? 1.f : __builtin_amdgcn_exp2f(mw - mm);
        ll += s_ml[i * per + r][1] * f;
#pragma unroll
        for (int e = 0; e < DV; ++e) o[e] += s_o[i * per + r][d0 + e] * f;
    }
    const int64_t row = r0 + r;
    const int tk = (int)(row / a.G), hd = hk * a.G + (int)(row - (int64_t)tk * a.G);
    T* op = (T*)a.O + (q.q0 + tk) * a.o_row + (int64_t)hd * a.o_head + d0;
    store_row<DV>(op, o, ll == 0.f ? 0.f : 1.f / ll);
}

// Joins the shares of a wide tile (bf16): 16 rows a block, 16 threads a row.
template <int DP, int SRC>
__global__ void __launch_bounds__(256)
prompt_join_kernel(PromptArgs a, int64_t slots) {
    constexpr int DV = DP / 16;
    const int R = a.rows, sub = blockIdx.x % (R / 16);
    const int64_t at = blockIdx.x / (R / 16), slot = at / a.Hk;
    const int hk = (int)(at % a.Hk);
    int s, tile;
    if (!prompt_slot<SRC>(a, a.G, R, slots, slot, s, tile)) return;
    const int64_t q0 = prompt_start(a.cu_q, s, a.q_tokens), rows = (prompt_start(a.cu_q, s + 1, a.q_tokens) - q0) * a.G;
    const int r = 16 * sub + (threadIdx.x >> 4), d0 = (threadIdx.x & 15) * DV;
    const int64_t row = (int64_t)tile * R + r;
    if (tile < 0 || row >= rows || d0 >= a.D) return;
    const float* part = a.part + (slot * a.splits * a.Hk + hk) * (int64_t)(R * (DP + 2));
    const int64_t next = (int64_t)a.Hk * (R * (DP + 2));
    float mm = NEG_INF, ll = 0.f, o[DV];
#pragma unroll
    for (int e = 0; e < DV; ++e) o[e] = 0.f;
#pragma unroll 4
    for (int i = 0; i < a.splits; ++i) mm = fmaxf(mm, part[i * next + R * DP + r]);
#pragma unroll 4
    for (int i = 0; i < a.splits; ++i) {
        const float* p = part + i * next;
        const float mw = p[R * DP + r], f = mw == mm ? 1.f : __builtin_amdgcn_exp2f(mw - mm);
        ll += p[R * DP + R + r] * f;
#pragma unroll
        for (int e = 0; e < DV; e += 4) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(p + (int64_t)r * DP + d0 + e);
#pragma unroll
            for (int x = 0; x < 4; ++x) o[e + x] += v[x] * f;
        }
    }
    const int tk = (int)(row / a.G), hd = hk * a.G + (int)(row - (int64_t)tk * a.G);
    uint16_t* op = (uint16_t*)a.O + (q0 + tk) * a.o_row + (int64_t)hd * a.o_head + d0;
    store_row<DV>(op, o, ll == 0.f ? 0.f : 1.f / ll);
}

int launch_prompt_join(const PromptArgs& a, int src, hipStream_t st) {
    const int64_t slots = prompt_slots(a, a.G, a.rows);
    const unsigned grid = (unsigned)(slots * a.Hk * (a.rows / 16));
    auto kernel = src == SRC_STORE ? a.D <= 64 ? prompt_join_kernel<64, SRC_STORE> : prompt_join_kernel<128, SRC_STORE>
                                   : a.D <= 64 ? prompt_join_kernel<64, SRC_PACKED> : prompt_join_kernel<128, SRC_PACKED>;
    kernel<<<grid, 256, 0, st>>>(a, slots);
    return check_launch("prompt_join_kernel");
}

template <typename T, int DP, int SRC, int DX, bool PAD = false>
static int launch_few_as(const PromptArgs& a, hipStream_t st) {
    prompt_few_kernel<T, DP, SRC, DX, PAD><<<(unsigned)a.blocks, 256, 0, st>>>(a);
    PS_TRY(check_launch("prompt_few_kernel"));
    if (a.unit == 0) return PSERVE_OK;
    prompt_meet_kernel<T, DP, SRC><<<(unsigned)a.blocks, 512, 0, st>>>(a);
    return check_launch("prompt_meet_kernel");
}
template <typename T, int SRC>
static int launch_few(const PromptArgs& a, hipStream_t st) {
    if constexpr (SRC == SRC_PACKED)            // (bf16: packed fp32 has launch_few_f32)
        if (a.D % 64) return a.D <= 64 ? launch_few_as<T, 64, SRC, 4, true>(a, st) : launch_few_as<T, 128, SRC, 8, true>(a, st);
    return a.D <= 64 ? launch_few_as<T, 64, SRC, 4>(a, st) : launch_few_as<T, 128, SRC, 8>(a, st);
}
static int launch_few_f32(const PromptArgs& a, hipStream_t st) {
    switch (a.D / 16) {
        case 1: return launch_few_as<float, 64, SRC_PACKED, 1>(a, st);
        case 2: return launch_few_as<float, 64, SRC_PACKED, 2>(a, st);
        case 3: return launch_few_as<float, 64, SRC_PACKED, 3>(a, st);
        case 4: return launch_few_as<float, 64, SRC_PACKED, 4>(a, st);
        case 5: return launch_few_as<float, 128, SRC_PACKED, 5>(a, st);
        case 6: return launch_few_as<float, 128, SRC_PACKED, 6>(a, st);
        case 7: return launch_few_as<float, 128, SRC_PACKED, 7>(a, st);
        default: return launch_few_as<float, 128, SRC_PACKED, 8>(a, st);
    }
}

int launch_prompt_few(const PromptArgs& a, int dtype, int src, hipStream_t st) {
    if (dtype == PSERVE_BF16) return src == SRC_STORE ? launch_few<uint16_t, SRC_STORE>(a, st) : launch_few<uint16_t, SRC_PACKED>(a, st);
    return src == SRC_STORE ? launch_few<float, SRC_STORE>(a, st) : launch_few_f32(a, st);
}

}  // namespace pserve
