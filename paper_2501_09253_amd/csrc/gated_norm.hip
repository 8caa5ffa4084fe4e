// Norms before and after a sub-layer with its gate and residual scale (pserve_gated_norm), gfx950.
//
//   y = skip_scale x + branch_scale gate_s (N_post(f) post_gain + post_bias)        the end of one sub-layer,
//   h = (N_pre(y) pre_gain + pre_bias) (1 + scale_s) + shift_s                      the beginning of the next,
//
// s the request of the row, N nothing, v / sqrt(mean v^2 + eps) or (v - mean) / sqrt(variance + eps).  Bound by memory: a row is read
// into registers once, both norms' sums are taken there (fp32; the variance from the deviations, a second walk over the registers), y
// is rounded where it is stored and only there.  h is rounded to the call's type or to 8-bit rows, whose blocks of 128 are sixteen lanes.
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

// The request of a row and the index of its vectors: the last s with cu[s] <= row, 64 places of the range looked at in one go.
// Where the starts do not ascend, any one; false: none, or one whose vectors are not there.
__device__ __forceinline__ bool norm_request(const NormArgs& a, int64_t row, int& s) {
    s = 0;
    if (a.cu) {
        const int lane = threadIdx.x & 63;
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
    }
    if (a.which) {
        s = a.which[s];
        if (s < 0 || s >= a.n) return false;
    }
    s = __builtin_amdgcn_readfirstlane(s);
    return true;
}

// The sum over the TPR threads of a row, in all of them, in a fixed order
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* s_part) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    if (TPR == 256) {
        __syncthreads();                        // (the sum before has been read)
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (s_part[0] + s_part[1]) + (s_part[2] + s_part[3]);
    }
    return v;
}

template <typename T, int TPR, int CH, bool VEC>
__global__ void __launch_bounds__(256)
gated_norm_kernel(NormArgs a) {
    __shared__ float s_part[4];
    const int t = threadIdx.x % TPR;
    const int64_t row = block_of_lines() * (256 / TPR) + threadIdx.x / TPR;
    if (row >= a.rows) return;
    int s;
    if (!norm_request(a, row, s)) return;
    const int C = a.C;
    auto get = [&](const T* p, int c, float (&v)[8]) {
        if (VEC) {
            if (8 * c < C) load8(p + 8 * c, v);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 8 * c + e < C ? load1(p + 8 * c + e) : 0.f;
        }
    };
    auto put = [&](T* p, int c, const float (&v)[8]) {
        if (VEC) {
            if (8 * c < C) store8(p + 8 * c, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (8 * c + e < C) store1(p + 8 * c + e, v[e]);
        }
    };
    auto in_row = [&](int c, int e) { return VEC ? 8 * c < C : 8 * c + e < C; };
    const float by = 1.f / (float)C;
    // what N multiplies by, after taking the mean off in place
    auto normed = [&](float (&v)[CH][8], int kind, float eps) -> float {
        if (kind == PSERVE_NORM_LAYER) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += v[i][e];
            const float mean = row_sum<TPR>(sum, s_part) * by;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = in_row(t + i * TPR, e) ? v[i][e] - mean : 0.f;
        }
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(v[i][e], v[i][e], sq);
        return 1.f / sqrtf(row_sum<TPR>(sq, s_part) * by + eps);
    };
    float v[CH][8], w[8];
    const T* xr = (const T*)a.x + row * a.xs;
    if (a.f) {
        const T* fr = (const T*)a.f + row * a.fs;
#pragma unroll
        for (int i = 0; i < CH; ++i) get(fr, t + i * TPR, v[i]);
        const float r = a.post != PSERVE_NORM_NONE ? normed(v, a.post, a.post_eps) : 1.f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = t + i * TPR;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= r;
            if (a.post_gain) {
                get((const T*)a.post_gain, c, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] *= w[e];
            }
            if (a.post_bias) {
                get((const T*)a.post_bias, c, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] += w[e];
            }
            if (a.gate) {
                get((const T*)a.gate + s * a.gate_s, c, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] *= w[e];
            }
            get(xr, c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = in_row(c, e) ? fmaf(a.branch, v[i][e], a.skip * w[e]) : 0.f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            get(xr, t + i * TPR, v[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= a.skip;
        }
    }
    if (a.y)
#pragma unroll
        for (int i = 0; i < CH; ++i) put((T*)a.y + row * a.ys, t + i * TPR, v[i]);
    if (!a.h && !a.v8) return;
    const float r = a.pre != PSERVE_NORM_NONE ? normed(v, a.pre, a.pre_eps) : 1.f;
    const int Kp = f8_width(C), Sp = f8_scales(C);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = t + i * TPR;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] *= r;
        if (a.pre_gain) {
            get((const T*)a.pre_gain, c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= w[e];
        }
        if (a.pre_bias) {
            get((const T*)a.pre_bias, c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] += w[e];
        }
        if (a.scale) {
            get((const T*)a.scale + s * a.scale_s, c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= 1.f + w[e];
        }
        if (a.shift) {
            get((const T*)a.shift + s * a.shift_s, c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] += w[e];
        }
        if (a.h) put((T*)a.h + row * a.hs, c, v[i]);
        if (a.v8 && 8 * c < Kp) {               // (sixteen lanes in step)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = in_row(c, e) ? v[i][e] : 0.f;
            const F8Scale z(lanes_max<16>(f8_largest(v[i])));
            *reinterpret_cast<q8_u32x2*>(a.v8 + row * Kp + 8 * c) = z.pack8(v[i]);
            if (c % 16 == 0) a.s8[row * Sp + c / 16] = (uint8_t)z.byte;
            if (c == 0)
                for (int b = Kp / 128; b < Sp; ++b) a.s8[row * Sp + b] = 127;
        }
    }
}

template <typename T, bool VEC>
static int launch_norm(const NormArgs& a, hipStream_t st) {
    const int chunks = (int)cdiv(a.C, 8);
    const dim3 waves = block_lines(cdiv(a.rows, 4)), rows = block_lines(a.rows);
    if (chunks <= 64) gated_norm_kernel<T, 64, 1, VEC><<<waves, 256, 0, st>>>(a);
    else if (chunks <= 128) gated_norm_kernel<T, 64, 2, VEC><<<waves, 256, 0, st>>>(a);
    else if (chunks <= 256) gated_norm_kernel<T, 256, 1, VEC><<<rows, 256, 0, st>>>(a);
    else if (chunks <= 512) gated_norm_kernel<T, 256, 2, VEC><<<rows, 256, 0, st>>>(a);
    else if (chunks <= 1024) gated_norm_kernel<T, 256, 4, VEC><<<rows, 256, 0, st>>>(a);
    else gated_norm_kernel<T, 256, 8, VEC><<<rows, 256, 0, st>>>(a);
    return check_launch("gated_norm_kernel");
}

}  // namespace pserve

extern "C" {

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
    bool vec = d->C % 8 == 0;
    for (const auto& r : rowed) {
        if (!r.p) continue;
        PS_REQUIRE(!((uintptr_t)r.p & (es - 1)), "%s: a buffer is not aligned to its type", who);
        PS_REQUIRE(r.stride >= 0 && r.stride < (1ll << 31) && (!r.row || d->rows == 1 || r.stride >= d->C), "%s: a stride of %lld elements (C = %d)", who, (long long)r.stride, d->C);
        vec = vec && !((uintptr_t)r.p & 15) && r.stride * es % 16 == 0;
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
    if (d->dtype == PSERVE_BF16) return vec ? launch_norm<uint16_t, true>(a, st) : launch_norm<uint16_t, false>(a, st);
    return vec ? launch_norm<float, true>(a, st) : launch_norm<float, false>(a, st);
}

}  // extern "C"
