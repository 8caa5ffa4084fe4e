// Norms before and after a sub-layer with its gate and residual scale (pserve_gated_norm), gfx950.
//
//   y = skip_scale x + branch_scale gate_s (N_post(f) post_gain + post_bias)        the end of one sub-layer,
//   h = (N_pre(y) pre_gain + pre_bias) (1 + scale_s) + shift_s                      the beginning of the next,
//
// s the request of the row, N nothing, v / sqrt(mean v^2 + eps) or (v - mean) / sqrt(variance + eps).  Bound by memory: a row is read
// into registers once, both norms' sums are taken there (fp32; the variance from the deviations, a second walk over the registers), y
// is rounded where it is stored and only there.  h is rounded to the call's type or to 8-bit rows, whose blocks of 128 are sixteen lanes.
// 12,544 x 1536, bf16, both norms, gate, scale and shift: 29 us, 5.2 TB/s (a copy: 5.0; part of the inputs comes from the last-level cache); into 8-bit rows 34
// (the rounding's instructions).  32 x 4096: 4.9, two sums' meetings behind the way to memory.
#include "f8.h"

using namespace pserve;

namespace pserve {

struct NormArgs {
    const void *x, *f, *post_gain, *post_bias, *gate, *pre_gain, *pre_bias, *scale, *shift;
    const int32_t *cu, *which;
    void *y, *h;
    uint8_t *v8, *s8;                           // 8-bit rows: numbers, scale bytes
    int64_t rows, xs, fs, ys, hs, gate_s, scale_s, shift_s;
    float skip, branch, post_eps, pre_eps;
    int32_t C, n, post, pre;
};

// The request of a row and the index of its vectors: the last s with cu[s] <= row.  Where the starts do not ascend, any one; false: none, or one whose
// vectors are not there.  WAVE: the row is a wavefront's, which looks at 64 places in one go; else a lane's own search
template <bool WAVE>
__device__ __forceinline__ bool norm_request(const NormArgs& a, int64_t row, int& s) {
    s = 0;
    if (a.cu) {
        const int lane = threadIdx.x & 63;
        if (WAVE && a.n < 64) {
            const uint64_t past = ~__ballot(lane <= a.n && a.cu[min(lane, a.n)] <= row);
            s = __ffsll((unsigned long long)past) - 2;          // (bit 63 is one of them, or n = 63 and the row is behind the last request)
            if (past == 0 || s < 0 || s >= a.n) return false;
        } else if (WAVE) {
            int lo = 0, len = a.n;
            for (;;) {
                const int step = (len + 63) / 64;
                const bool le = lane * step < len && a.cu[lo + lane * step] <= row;
                const uint64_t past = ~__ballot(le);
                const int count = past ? __ffsll((unsigned long long)past) - 1 : 64;
                if (count == 0) return false;
                lo += (count - 1) * step;
                len = min(step, len - (count - 1) * step);
                if (step == 1) break;
            }
            s = lo;
            if (row >= a.cu[s + 1]) return false;
        } else {
            int lo = 0, hi = a.n;                               // cu[lo] <= row < cu[hi], where the ends hold
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (a.cu[mid] <= row) lo = mid;
                else hi = mid;
            }
            s = lo;
            if (row < a.cu[s] || row >= a.cu[s + 1]) return false;
        }
    }
    if (a.which) {
        s = a.which[s];
        if (s < 0 || s >= a.n) return false;
    }
    if (WAVE) s = __builtin_amdgcn_readfirstlane(s);
    return true;
}

// The sum over the threads of a row, in all of them, in a fixed order: TPR neighbouring lanes, or (TPR = 0) a block
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* s_part) {
    v = lanes_sum<TPR ? TPR : 64>(v);
    if (TPR == 0) {
        __syncthreads();                        // (the sum before has been read)
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s_part[0];
        for (int i = 1; i < (int)blockDim.x / 64; ++i) v += s_part[i];
    }
    return v;
}

// TPR threads a row (0: a block), CH chunks of 16 bytes a thread; EVEN: whole chunks
template <typename T, int TPR, int CH, bool EVEN>
__global__ void __launch_bounds__(TPR ? 256 : 1024)
gated_norm_kernel(NormArgs a) {
    __shared__ float s_part[16];
    const int span = TPR ? TPR : blockDim.x, t = TPR ? (int)threadIdx.x % TPR : (int)threadIdx.x;
    const int64_t row = TPR ? block_of_lines() * (256 / TPR) + threadIdx.x / TPR : block_of_lines();
    if (row >= a.rows) return;
    const int C = a.C;
    constexpr int V = 16 / sizeof(T);           // values of a chunk
    typedef typename AnyPiece<T>::type Any;
    auto fetch = [&](const T* p, int c, u32x4& r) {
        if (EVEN ? V * c < C : V * c + V <= C) {
            r = *reinterpret_cast<const Any*>(p + V * c);
        } else {
            T v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = !EVEN && V * c + e < C ? p[V * c + e] : T(0);
            __builtin_memcpy(&r, v, sizeof r);
        }
    };
    auto values = [&](const u32x4& r, float (&v)[V]) {
        T x[V];
        __builtin_memcpy(x, &r, sizeof r);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = load1(x + e);
    };
    auto get = [&](const T* p, int c, float (&v)[V]) {
        u32x4 r;
        fetch(p, c, r);
        values(r, v);
    };
    auto put = [&](T* p, int c, const float (&v)[V]) {
        T o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) store1(o + e, v[e]);
        if (EVEN ? V * c < C : V * c + V <= C) {
            u32x4 r;
            __builtin_memcpy(&r, o, sizeof r);
            __builtin_nontemporal_store(r, reinterpret_cast<Any*>(p + V * c));
        } else if (!EVEN) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (V * c + e < C) p[V * c + e] = o[e];
        }
    };
    auto in_row = [&](int c, int e) { return EVEN ? V * c < C : V * c + e < C; };
    const float by = 1.f / (float)C;
    // what N multiplies by, after taking the mean off in place
    auto normed = [&](float (&v)[CH][V], int kind, float eps) -> float {
        if (kind == PSERVE_NORM_LAYER) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) sum += v[i][e];
            const float mean = row_sum<TPR>(sum, s_part) * by;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) v[i][e] = in_row(t + i * span, e) ? v[i][e] - mean : 0.f;
        }
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) sq = fmaf(v[i][e], v[i][e], sq);
        return 1.f / sqrtf(row_sum<TPR>(sq, s_part) * by + eps);
    };
    // The row comes in beside the search for its request, and with it known the vectors beside the sums
    float v[CH][V], w[V];
    u32x4 xw[CH], fw[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) fetch((const T*)a.x + row * a.xs, t + i * span, xw[i]);
    if (a.f)
#pragma unroll
        for (int i = 0; i < CH; ++i) fetch((const T*)a.f + row * a.fs, t + i * span, fw[i]);
    int s;
    if (!norm_request<(TPR == 0 || TPR == 64)>(a, row, s)) return;
    u32x4 gw[2][CH];
    const T *first[2] = {(const T*)a.post_gain, a.gate ? (const T*)a.gate + s * a.gate_s : nullptr};
    const T *second[2] = {a.scale ? (const T*)a.scale + s * a.scale_s : nullptr, a.shift ? (const T*)a.shift + s * a.shift_s : nullptr};
    auto ahead = [&](const T* const (&from)[2]) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (from[k])
#pragma unroll
                for (int i = 0; i < CH; ++i) fetch(from[k], t + i * span, gw[k][i]);
    };
    if (a.f) {
        ahead(first);
#pragma unroll
        for (int i = 0; i < CH; ++i) values(fw[i], v[i]);
        const float r = a.post != PSERVE_NORM_NONE ? normed(v, a.post, a.post_eps) : 1.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = t + i * span;
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] *= r;
            if (a.post_gain) {
                values(gw[0][i], w);
#pragma unroll
                for (int e = 0; e < V; ++e) v[i][e] *= w[e];
            }
            if (a.post_bias) {
                get((const T*)a.post_bias, c, w);
#pragma unroll
                for (int e = 0; e < V; ++e) v[i][e] += w[e];
            }
            if (a.gate) {
                values(gw[1][i], w);
#pragma unroll
                for (int e = 0; e < V; ++e) v[i][e] *= w[e];
            }
            values(xw[i], w);
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] = in_row(c, e) ? fmaf(a.branch, v[i][e], a.skip * w[e]) : 0.f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            values(xw[i], v[i]);
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] *= a.skip;
        }
    }
    if (a.y)
#pragma unroll
        for (int i = 0; i < CH; ++i) put((T*)a.y + row * a.ys, t + i * span, v[i]);
    if (!a.h && !a.v8) return;
    ahead(second);
    const float r = a.pre != PSERVE_NORM_NONE ? normed(v, a.pre, a.pre_eps) : 1.f;
    const int Kp = f8_width(C), Sp = f8_scales(C);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = t + i * span;
#pragma unroll
        for (int e = 0; e < V; ++e) v[i][e] *= r;
        if (a.pre_gain) {
            get((const T*)a.pre_gain, c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] *= w[e];
        }
        if (a.pre_bias) {
            get((const T*)a.pre_bias, c, w);
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] += w[e];
        }
        if (a.scale) {
            values(gw[0][i], w);
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] *= 1.f + w[e];
        }
        if (a.shift) {
            values(gw[1][i], w);
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] += w[e];
        }
        if (a.h) put((T*)a.h + row * a.hs, c, v[i]);
        if (a.v8 && V * c < Kp) {               // (the lanes of a block of 128 in step)
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] = in_row(c, e) ? v[i][e] : 0.f;
            constexpr int LANES = 128 / V;
            uint32_t m = lanes_max<16>(f8_largest(v[i]));
            if (LANES == 32) m = max_16_apart(m);
            F8Scale(m).pack(v[i], a.v8 + row * Kp + V * c);
            if (c % LANES == 0) a.s8[f8_scale_at(a.rows, row, c / LANES)] = (uint8_t)F8Scale(m).byte;
            if (c == 0)
                for (int b = Kp / 128; b < Sp; ++b) a.s8[f8_scale_at(a.rows, row, b)] = 127;
        }
    }
}

template <typename T, int TPR, int CH, bool EVEN>
static int launch_norm_as(const NormArgs& a, hipStream_t st) {
    const int block = TPR ? 256 : (int)cdiv(cdiv(a.C, 16 / sizeof(T)), 64 * CH) * 64;
    gated_norm_kernel<T, TPR, CH, EVEN><<<block_lines(TPR ? cdiv(a.rows, 256 / (TPR ? TPR : 1)) : a.rows), block, 0, st>>>(a);
    return check_launch("gated_norm_kernel");
}
// A row is a wavefront's, or a part of one, where its 16-byte chunks are that many lanes, and a block's else.  Outputs go past the caches (12,544 x 1536,
// bf16, y and h: 39 -> 32 us, 4.9 TB/s; 300,000 x 64 41 -> 32); 8-bit rows do not: the product reads them next.
// 10 x threads of a row (0: a block) + chunks of a thread
static int norm_form(size_t size, int64_t rows, int32_t C, bool rows8) {
    const int chunks = (int)cdiv(C, 16 / (int)size), least = rows8 ? F8_BLOCK * (int)size / 16 : 1;                 // (8-bit rows have whole blocks)
    if (chunks <= 8 && least <= 8) return 81;
    if (chunks <= 16 && least <= 16) return 161;
    if (chunks <= 32) return 321;
    if (chunks <= 64) return 641;
    // (60,000 x 640, bf16: 91 us by blocks of 128, 75 by wavefronts; 500 x 640 the other way round)
    if (chunks <= 128 && rows >= 8192) return 642;
    return chunks <= 512 ? 1 : chunks <= 2048 ? 2 : 4;
}
template <typename T, bool EVEN>
static int launch_norm(const NormArgs& a, hipStream_t st) {
    const int form = norm_form(sizeof(T), a.rows, a.C, a.v8 != nullptr);
    if constexpr (sizeof(T) == 4)               // (bf16: up to 2048 chunks)
        if (form == 4) return launch_norm_as<T, 0, 4, EVEN>(a, st);
    switch (form) {
        case 81: return launch_norm_as<T, 8, 1, EVEN>(a, st);
        case 161: return launch_norm_as<T, 16, 1, EVEN>(a, st);
        case 321: return launch_norm_as<T, 32, 1, EVEN>(a, st);
        case 641: return launch_norm_as<T, 64, 1, EVEN>(a, st);
        case 642: return launch_norm_as<T, 64, 2, EVEN>(a, st);
        case 1: return launch_norm_as<T, 0, 1, EVEN>(a, st);
        default: return launch_norm_as<T, 0, 2, EVEN>(a, st);
    }
}

}  // namespace pserve

extern "C" {

// For tests (not in the header): the form of a call, see norm_form
int pserve_test_gated_norm_form(int dtype, int64_t rows, int32_t C, int rows8) { return norm_form(dtype_size(dtype), rows, C, rows8 != 0); }

int pserve_gated_norm(const pserve_gated_norm_desc* d, const pserve_gated_norm_buffers* b, void* stream) {
    static const char who[] = "pserve_gated_norm";
    PS_REQUIRE(d && b, "%s: NULL argument", who);
    PS_REQUIRE(d->dtype == PSERVE_F32 || d->dtype == PSERVE_BF16, "%s: unknown dtype %d", who, d->dtype);
    PS_REQUIRE(d->C > 0 && d->C <= PSERVE_GATED_NORM_MAX_C, "%s: %d channels (1 .. %d)", who, d->C, PSERVE_GATED_NORM_MAX_C);
    PS_REQUIRE(d->n > 0, "%s: need n > 0 requests", who);
    for (int kind : {d->post_norm, d->pre_norm})
        PS_REQUIRE(kind == PSERVE_NORM_NONE || kind == PSERVE_NORM_RMS || kind == PSERVE_NORM_LAYER, "%s: unknown norm %d", who, kind);
    for (float eps : {d->post_eps, d->pre_eps}) PS_REQUIRE(eps >= 0.f && eps <= 3e38f, "%s: eps must be a number from 0", who);
    for (float f : {d->skip_scale, d->branch_scale}) PS_REQUIRE(f >= -3.4e38f && f <= 3.4e38f, "%s: a scale that is not finite", who);
    PS_REQUIRE(d->rows >= 0 && d->rows < (1ll << 31), "%s: %lld rows (fewer than 2^31)", who, (long long)d->rows);
    PS_REQUIRE(b->cu_rows || d->n == 1, "%s: %d requests without cu_rows", who, d->n);
    if (d->rows == 0) return PSERVE_OK;
    PS_REQUIRE(b->f || (d->post_norm == PSERVE_NORM_NONE && !b->post_gain && !b->post_bias && !b->gate), "%s: the end of a sub-layer without its output f", who);
    const bool next = b->h || b->rows8;
    PS_REQUIRE(next || (d->pre_norm == PSERVE_NORM_NONE && !b->pre_gain && !b->pre_bias && !b->scale && !b->shift), "%s: the beginning of a sub-layer without h", who);
    PS_REQUIRE(!(b->h && b->rows8), "%s: h and rows8 at once", who);
    PS_REQUIRE(b->x && (b->y || next), "%s: NULL buffer", who);
    struct { const void* p; int64_t stride; bool row; } rowed[] = {{b->x, d->x_stride, true}, {b->f, d->f_stride, true}, {b->y, d->y_stride, true}, {b->h, d->h_stride, true},
                                                                   {b->gate, d->gate_stride, false}, {b->scale, d->scale_stride, false}, {b->shift, d->shift_stride, false},
                                                                   {b->post_gain, d->C, false}, {b->post_bias, d->C, false}, {b->pre_gain, d->C, false}, {b->pre_bias, d->C, false}};
    const int64_t es = (int64_t)dtype_size(d->dtype);
    for (const auto& r : rowed) {
        if (!r.p) continue;
        PS_REQUIRE(!((uintptr_t)r.p & (es - 1)), "%s: a buffer is not aligned to its type", who);
        PS_REQUIRE(r.stride >= 0 && r.stride < (1ll << 31) && (!r.row || d->rows == 1 || r.stride >= d->C), "%s: a stride of %lld elements (C = %d)", who, (long long)r.stride, d->C);
    }
    PS_REQUIRE(!((uintptr_t)b->rows8 & 15), "%s: rows8 is not 16-byte aligned", who);
    NormArgs a{};
    a.x = b->x; a.f = b->f; a.post_gain = b->post_gain; a.post_bias = b->post_bias; a.gate = b->gate;
    a.pre_gain = b->pre_gain; a.pre_bias = b->pre_bias; a.scale = b->scale; a.shift = b->shift;
    a.cu = b->cu_rows; a.which = b->which; a.y = b->y; a.h = b->h;
    if (b->rows8) {
        a.v8 = (uint8_t*)b->rows8;
        a.s8 = a.v8 + (size_t)d->rows * f8_width(d->C);
    }
    a.rows = d->rows; a.xs = d->x_stride; a.fs = d->f_stride; a.ys = d->y_stride; a.hs = d->h_stride;
    a.gate_s = d->gate_stride; a.scale_s = d->scale_stride; a.shift_s = d->shift_stride;
    a.skip = d->skip_scale; a.branch = d->branch_scale; a.post_eps = d->post_eps; a.pre_eps = d->pre_eps;
    a.C = d->C; a.n = d->n; a.post = d->post_norm; a.pre = d->pre_norm;
    hipStream_t st = (hipStream_t)stream;
    if (d->dtype == PSERVE_BF16) return d->C % 8 == 0 ? launch_norm<uint16_t, true>(a, st) : launch_norm<uint16_t, false>(a, st);
    return d->C % 4 == 0 ? launch_norm<float, true>(a, st) : launch_norm<float, false>(a, st);
}

}  // extern "C"
