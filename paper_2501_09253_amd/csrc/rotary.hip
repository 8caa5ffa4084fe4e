// Rotary positions with several axes (pserve_rotary_*, pserve_plan_positions), gfx950.
//
//   theta_p = pos[t][axis_p] * freq_p,   (a, b) -> (a cos theta_p - b sin theta_p, a sin theta_p + b cos theta_p)
//
// for each pair p of values of a head.  Bound by memory: every value is read and written once.  The angles are a token's, whatever its
// heads are: a block computes those of its tokens once, into LDS, then walks its tokens' heads in 16-byte pieces.
// An angle is taken in revolutions, in 64 bits (positions reach 2^24, and 32 bits leave a position of 2^17 with an angle off by 2^-7); the
// fraction of a revolution is rounded to fp32, at most 2^-26 off: 2^-23.3 radians.  2 pi, the quotient of a frequency by it and the product are rounded to 64 bits:
// together at most 3 * 2^-53 of an angle (1.12 * 2^-52 seen), 2^-22 radians at 2^29.
// bf16, heads of 64: 12,544 tokens of 48, neighbours paired, 29 us (5.3 TB/s, part of the values from the last-level cache), 131,072 tokens of 20, halves
// paired, 141 (4.8); a large copy runs at 5.0.  48 tokens of 40 heads of 128: 4.7, the way to positions, values and back.
#include "f8.h"

using namespace pserve;

struct pserve_rotary_s {
    int32_t axes = 0, pairs = 0, layout = 0;
    int device = 0;
    double* freq = nullptr;                     // [pairs] revolutions a unit of position
    int32_t* axis = nullptr;                    // [pairs]
    pserve::DevicePool pool;
};

namespace pserve {

struct RotaryArgs {
    const void *q, *k;
    void *q_out, *k_out;
    const float* pos;                           // [tokens][axes]
    const double* freq;
    const int32_t* axis;
    int64_t tokens, qs[2], ks[2], qo[2], ko[2];
    int32_t heads, kv_heads, D, P, axes, TB;    // TB: tokens of a block
    int32_t lines;                              // store instructions write whole runs of 128 bytes
    int32_t keep;                               // in place: what is not turned stays
};

// cosine and sine of the angles of a block's tokens: pair p of token t at [t * P + p]
__device__ __forceinline__ void rotary_angles(const RotaryArgs& a, int64_t t0, int nt, float2* cs) {
    for (int i = threadIdx.x; i < nt * a.P; i += blockDim.x) {
        const int t = i / a.P, p = i - t * a.P;
        const double turn = (double)a.pos[(t0 + t) * a.axes + a.axis[p]] * a.freq[p];
        const float f = (float)(turn - rint(turn));             // -1/2 .. 1/2 of a revolution
        float s, c;
        sincospif(2.f * f, &s, &c);
        cs[i] = make_float2(c, s);
    }
}

// n / d for n * d < 2^32, by the rounded-up reciprocal
struct Divisor {
    uint32_t d, m;
    explicit Divisor(uint32_t d_) : d(d_), m(d_ > 1 ? (uint32_t)(((1ull << 32) + d_ - 1) / d_) : 0) {}
    __device__ __forceinline__ int operator()(int n) const { return d > 1 ? (int)__umulhi((uint32_t)n, m) : n; }
};

// An item is K pieces of 16 bytes of a head, at any element's address, V values each.  HALF: two, the values of V pairs, from p and P + p on, then pieces of
// what is copied, half of that apart.  NEXT: one, of whole pairs, turned or copied.
// A block's items are numbered line by line (token, head); a thread asks for its first IT items before the angles are formed, so the two ways to
// memory overlap.
template <typename T, bool HALF, int IT>
__global__ void __launch_bounds__(256, 6)
rotary_kernel(RotaryArgs a, Divisor items, Divisor heads) {
    extern __shared__ float2 s_turn[];
    constexpr int V = 16 / sizeof(T), K = HALF ? 2 : 1;
    typedef typename AnyPiece<T>::type Any;
    const int64_t t0 = block_of_lines() * a.TB;
    if (t0 >= a.tokens) return;
    const int nt = (int)min((int64_t)a.TB, a.tokens - t0), total = nt * (int)(heads.d * items.d);
    const int turned = HALF ? (a.P + V - 1) / V : 0, last = a.keep ? 2 * a.P : a.D, begin = HALF ? 2 * a.P : 0;     // copied (NEXT: all) values: begin .. last - 1
    const int apart = (int)items.d - turned;                    // between the pieces of an item of those
    const T* in;
    T* out;
    int cs, at[K], len[K];                                      // the token's angles; where the pieces are, and how many values
    bool pairs;                                                 // (HALF) an item of pairs
    auto place = [&](int i) {
        const int line = items(i), c = i - line * (int)items.d, t = heads(line), h = line - t * (int)heads.d, hk = h - a.heads;
        if (hk < 0) {
            in = (const T*)a.q + (t0 + t) * a.qs[0] + h * a.qs[1];
            out = (T*)a.q_out + (t0 + t) * a.qo[0] + h * a.qo[1];
        } else {
            in = (const T*)a.k + (t0 + t) * a.ks[0] + hk * a.ks[1];
            out = (T*)a.k_out + (t0 + t) * a.ko[0] + hk * a.ko[1];
        }
        cs = t * a.P;
        pairs = HALF && c < turned;
        if (pairs) {
            at[0] = c * V;
            at[K - 1] = a.P + c * V;
            len[0] = len[K - 1] = min(V, a.P - c * V);
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                at[k] = begin + (c - turned + k * apart) * V;
                len[k] = max(0, min(V, last - at[k]));
            }
        }
    };
    auto load = [&](int i, u32x4 (&x)[K]) {
        place(i);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (len[k] == V) x[k] = *reinterpret_cast<const Any*>(in + at[k]);
            else {
                T v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = e < len[k] ? in[at[k] + e] : T(0);
                __builtin_memcpy(&x[k], v, sizeof v);
            }
        }
    };
    auto finish = [&](int i, u32x4 (&x)[K]) {
        place(i);
        T v[K][V];
        __builtin_memcpy(v, x, sizeof v);
        if constexpr (HALF) {
            if (pairs)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float2 t = s_turn[cs + min(at[0] + e, a.P - 1)];
                    const float p = load1(&v[0][e]), q = load1(&v[K - 1][e]);
                    store1(&v[0][e], p * t.x - q * t.y);
                    store1(&v[K - 1][e], p * t.y + q * t.x);
                }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    const int pair = (at[k] + e) >> 1;
                    const float2 t = s_turn[cs + min(pair, a.P - 1)];
                    const float p = load1(&v[k][e]), q = load1(&v[k][e + 1]);
                    T o[2];
                    store1(o, p * t.x - q * t.y);
                    store1(o + 1, p * t.y + q * t.x);
                    v[k][e] = pair < a.P ? o[0] : v[k][e];
                    v[k][e + 1] = pair < a.P ? o[1] : v[k][e + 1];
                }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (len[k] == V) {
                u32x4 o;
                __builtin_memcpy(&o, v[k], sizeof o);
                store_piece(out + at[k], o, a.lines);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e < len[k]) out[at[k] + e] = v[k][e];
            }
        }
    };
    u32x4 held[IT][K];
#pragma unroll
    for (int j = 0; j < IT; ++j)
        if (threadIdx.x + 256 * j < total) load(threadIdx.x + 256 * j, held[j]);
    rotary_angles(a, t0, nt, s_turn);
    __syncthreads();
#pragma unroll
    for (int j = 0; j < IT; ++j)
        if (threadIdx.x + 256 * j < total) finish(threadIdx.x + 256 * j, held[j]);
    for (int i = threadIdx.x + 256 * IT; i < total; i += 256) {
        load(i, held[0]);
        finish(i, held[0]);
    }
}

template <typename T>
static int launch_rotary(const RotaryArgs& in, int layout, hipStream_t st) {
    constexpr int V = 16 / sizeof(T);
    RotaryArgs a = in;
    const bool half = layout == PSERVE_PAIR_HALF;
    const int H = a.heads + a.kv_heads, rest = (a.keep ? 2 * a.P : a.D) - (half ? 2 * a.P : 0), items = half ? (int)cdiv(a.P, V) + (int)cdiv(rest, 2 * V) : (int)cdiv(rest, V);
    const int each = half ? 4 : 8;              // items of a thread
    // that many, but 512 blocks where the tokens give them; angles of a block: up to 32 KB
    a.TB = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(256 * each / (H * items), cdiv(a.tokens, 512)), 4096 / a.P));
    // Runs of 128 bytes go past the caches (12,544 tokens x 48 heads of 64, neighbours paired, bf16: 44 -> 35 us; runs of 64, 131,072 x 20 heads of 64, would take 150 for 143)
    auto line = [&](const void* p, const int64_t* s, int n) {
        return !((uintptr_t)p & 63) && (a.tokens == 1 || s[0] * (int64_t)sizeof(T) % 64 == 0) && (n == 1 || s[1] * (int64_t)sizeof(T) % 64 == 0);
    };
    a.lines = (half ? a.P : a.D) * (int)sizeof(T) % 128 == 0 && line(a.q_out, a.qo, a.heads) && (!a.kv_heads || line(a.k_out, a.ko, a.kv_heads));
    const dim3 grid = block_lines(cdiv(a.tokens, a.TB));
    const size_t lds = (size_t)a.TB * a.P * sizeof(float2);
    if (half) rotary_kernel<T, true, 4><<<grid, 256, lds, st>>>(a, Divisor(items), Divisor(H));
    else rotary_kernel<T, false, 8><<<grid, 256, lds, st>>>(a, Divisor(items), Divisor(H));
    return check_launch("rotary_kernel");
}

// ---- positions of a plan's tokens
struct PlanPosArgs {
    const int32_t *owner, *rc, *perm;
    const float* frame;
    float start[3], step[3];
    float* pos;
    int64_t T;
    int32_t S, ph, pw, text_len;
};
__global__ void __launch_bounds__(256)
plan_positions_kernel(PlanPosArgs a) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t >= a.T) return;
    const int p = (int)(t / a.S), r = (int)(t - (int64_t)p * a.S), row = a.rc[2 * p], col = a.rc[2 * p + 1];
    float* o = a.pos + 3 * t;
    if (row < 0) {                                              // text patch `col` of its request
        const int64_t j = (int64_t)col * a.S + r;
#pragma unroll
        for (int i = 0; i < 3; ++i) o[i] = j < a.text_len ? a.start[i] + (float)j * a.step[i] : 0.f;
        return;
    }
    const int y = r / a.pw, x = r - y * a.pw;
    o[0] = a.frame ? a.frame[a.perm[a.owner[p]]] : 0.f;
    o[1] = (float)(row * a.ph + y);
    o[2] = (float)(col * a.pw + x);
}

}  // namespace pserve

extern "C" {

int pserve_rotary_create(int32_t axes, int32_t pairs, const int32_t* axis, const double* freq, int layout, void* stream, pserve_rotary_t** out) {
    static const char who[] = "pserve_rotary_create";
    PS_REQUIRE(out, "%s: out is NULL", who);
    *out = nullptr;
    PS_REQUIRE(axis && freq, "%s: NULL argument", who);
    PS_REQUIRE(axes >= 1 && axes <= 8, "%s: %d axes (1 .. 8)", who, axes);
    PS_REQUIRE(pairs >= 1 && pairs <= 256, "%s: %d pairs (1 .. 256)", who, pairs);
    PS_REQUIRE(layout == PSERVE_PAIR_HALF || layout == PSERVE_PAIR_NEXT, "%s: unknown layout %d", who, layout);
    for (int i = 0; i < pairs; ++i) {
        PS_REQUIRE(axis[i] >= 0 && axis[i] < axes, "%s: axis %d of pair %d (%d axes)", who, axis[i], i, axes);
        PS_REQUIRE(freq[i] >= -1e9 && freq[i] <= 1e9, "%s: the frequency of pair %d is not finite or beyond 1e9", who, i);
    }
    return guarded(who, [&]() -> int {
        std::unique_ptr<pserve_rotary_t> op(new pserve_rotary_t());
        op->axes = axes; op->pairs = pairs; op->layout = layout;
        PS_CHECK_HIP(hipGetDevice(&op->device));
        PS_TRY(op->pool.alloc_t(&op->freq, pairs));
        PS_TRY(op->pool.alloc_t(&op->axis, pairs));
        std::vector<double> turns(pairs);
        for (int i = 0; i < pairs; ++i) turns[i] = freq[i] / 6.283185307179586476925286766559;
        hipStream_t st = (hipStream_t)stream;
        PS_CHECK_HIP(hipMemcpyAsync(op->freq, turns.data(), pairs * sizeof(double), hipMemcpyHostToDevice, st));
        PS_CHECK_HIP(hipMemcpyAsync(op->axis, axis, pairs * sizeof(int32_t), hipMemcpyHostToDevice, st));
        PS_CHECK_HIP(hipStreamSynchronize(st));
        *out = op.release();
        return PSERVE_OK;
    });
}

void pserve_rotary_free(pserve_rotary_t* op) { delete op; }

int pserve_rotary_forward(const pserve_rotary_t* op, const pserve_rotary_desc* d, const float* pos, const void* q, const void* k, void* q_out,
                          void* k_out, void* stream) {
    static const char who[] = "pserve_rotary_forward";
    PS_REQUIRE(op && d, "%s: NULL argument", who);
    PS_REQUIRE(d->dtype == PSERVE_F32 || d->dtype == PSERVE_BF16, "%s: unknown dtype %d", who, d->dtype);
    PS_REQUIRE(d->heads > 0 && d->kv_heads >= 0 && d->heads <= 4096 && d->kv_heads <= 4096, "%s: %d and %d heads (1 .. 4096, 0 .. 4096)", who, d->heads, d->kv_heads);
    PS_REQUIRE(d->head_dim >= 2 * op->pairs && d->head_dim <= 512, "%s: head_dim %d (%d pairs; up to 512)", who, d->head_dim, op->pairs);
    PS_REQUIRE(d->tokens >= 0 && d->tokens < (1ll << 31), "%s: %lld tokens (fewer than 2^31)", who, (long long)d->tokens);
    const int64_t* strides[4] = {d->q_stride, d->q_out_stride, d->k_stride, d->k_out_stride};
    for (int i = 0; i < (d->kv_heads ? 4 : 2); ++i)
        for (int j = 0; j < 2; ++j)
            PS_REQUIRE(strides[i][j] >= 0 && strides[i][j] < (1ll << 31), "%s: a stride of %lld elements", who, (long long)strides[i][j]);
    if (d->tokens == 0) return PSERVE_OK;
    PS_REQUIRE(pos && q && q_out && (!d->kv_heads || (k && k_out)), "%s: NULL buffer", who);
    const uintptr_t es = dtype_size(d->dtype);
    PS_REQUIRE(!(((uintptr_t)q | (uintptr_t)q_out | (d->kv_heads ? (uintptr_t)k | (uintptr_t)k_out : 0)) & (es - 1)) && !((uintptr_t)pos & 3),
               "%s: a buffer is not aligned to its type", who);
    int dev;
    PS_CHECK_HIP(hipGetDevice(&dev));
    PS_REQUIRE(dev == op->device, "%s: the frequencies are on device %d, the current one is %d", who, op->device, dev);
    RotaryArgs a{};
    a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out; a.pos = pos; a.freq = op->freq; a.axis = op->axis;
    a.tokens = d->tokens; a.heads = d->heads; a.kv_heads = d->kv_heads; a.D = d->head_dim; a.P = op->pairs; a.axes = op->axes;
    for (int j = 0; j < 2; ++j) {
        a.qs[j] = d->q_stride[j]; a.qo[j] = d->q_out_stride[j];
        a.ks[j] = d->k_stride[j]; a.ko[j] = d->k_out_stride[j];
    }
    a.keep = q == q_out && (!d->kv_heads || k == k_out);
    hipStream_t st = (hipStream_t)stream;
    return d->dtype == PSERVE_BF16 ? launch_rotary<uint16_t>(a, op->layout, st) : launch_rotary<float>(a, op->layout, st);
}

int pserve_plan_positions(const pserve_plan_t* plan, const float* frame, const float* text, float* pos, void* stream) {
    static const char who[] = "pserve_plan_positions";
    PS_REQUIRE(plan && pos, "%s: NULL argument", who);
    PlanPosArgs a{};
    a.owner = plan->d_tab[PSERVE_TAB_PATCH_OWNER]; a.rc = plan->d_tab[PSERVE_TAB_PATCH_RC]; a.perm = plan->d_tab[PSERVE_TAB_PERM];
    a.frame = frame; a.pos = pos; a.T = plan->T; a.S = plan->S; a.ph = plan->ph; a.pw = plan->pw; a.text_len = plan->text_len;
    for (int i = 0; i < 3; ++i) {
        a.start[i] = text ? text[i] : 0.f;
        a.step[i] = text ? text[3 + i] : 0.f;
    }
    plan_positions_kernel<<<(unsigned)cdiv(a.T, 256), 256, 0, (hipStream_t)stream>>>(a);
    return check_launch("plan_positions_kernel");
}

}  // extern "C"
