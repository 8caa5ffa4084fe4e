// Arguments and device pieces shared by the kernels of the prompt attention.
#pragma once

#include "kv8.h"
#include "quant8.h"

namespace pserve {

struct PromptArgs {
    const void *Q, *K, *V;              // SRC_PACKED: K and V; SRC_STORE: the four pointers of the store below
    void* O;
    const int8_t *k8, *v8;              // [places][Hk][D]
    const float *k_scale, *v_scale;     // [places][Hk]
    const int32_t *cu_q, *cu_k;         // [n + 1]
    const int32_t *key_len, *table;     // SRC_STORE: [n], [n][max_pages]
    float* part;                        // partial results of the key shares
    int64_t q_tokens, k_tokens;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;     // strides in elements
    int32_t n, H, Hk, G, D, causal, rows, splits;      // rows of a tile, shares of its keys
    int32_t max_pages, page_shift, pages;
    float scale2;                       // scale * log2(e)
};
enum { SRC_PACKED = 0, SRC_STORE = 1 };

// queries and keys of sequence s.  What the device arrays hold is cut to the tensors' sizes: no value of them leads outside
struct PromptSeq {
    int64_t q0, k0;
    int32_t Lq, Lk;
};
__device__ __forceinline__ int64_t prompt_start(const int32_t* cu, int s, int64_t tokens) {
    const int64_t c = cu[s];
    return c < 0 ? 0 : c > tokens ? tokens : c;
}
template <int SRC>
__device__ __forceinline__ PromptSeq prompt_seq(const PromptArgs& a, int s) {
    PromptSeq q;
    q.q0 = prompt_start(a.cu_q, s, a.q_tokens);
    q.Lq = (int32_t)max((int64_t)0, prompt_start(a.cu_q, s + 1, a.q_tokens) - q.q0);
    if constexpr (SRC == SRC_PACKED) {
        q.k0 = prompt_start(a.cu_k, s, a.k_tokens);
        q.Lk = (int32_t)max((int64_t)0, prompt_start(a.cu_k, s + 1, a.k_tokens) - q.k0);
    } else {
        q.k0 = 0;
        const int64_t most = (int64_t)a.max_pages << a.page_shift;
        q.Lk = (int32_t)max((int64_t)0, min((int64_t)a.key_len[s], most));
    }
    return q;
}
// Tiles of R rows over sequences of cu_q[s + 1] - cu_q[s] tokens of G rows each, without a table made by the host: sequence s has
// the slots from floor(cu_q[s] G / R) + s on, at least as many as it has tiles.  false: no sequence's.
__device__ __forceinline__ bool prompt_slot(const PromptArgs& a, int G, int R, int64_t slot, int& s, int& tile) {
    const int lane = threadIdx.x & 63;
    int count = 0;
    for (int b = 0; b < a.n; b += 64) {
        const int i = b + lane;
        const bool le = i < a.n && prompt_start(a.cu_q, i, a.q_tokens) * G / R + i <= slot;
        const uint64_t m = __ballot(le);
        count += __popcll(m);
        if (m != ~0ull) break;
    }
    if (count == 0) return false;
    s = __builtin_amdgcn_readfirstlane(count - 1);
    const int64_t t = slot - (prompt_start(a.cu_q, s, a.q_tokens) * G / R + s);
    tile = (int)t;
    return true;
}
inline int64_t prompt_slots(const PromptArgs& a, int G, int R) { return a.q_tokens * G / R + a.n; }

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

// two whole numbers of a dword of four (bytes 2 h, 2 h + 1) as a pair of bf16: exact, 7 bits and a sign
__device__ __forceinline__ uint32_t bf16_of_i8(uint32_t w, int h) {
    const float lo = (float)(int8_t)(w >> (16 * h)), hi = (float)(int8_t)(w >> (16 * h + 8));
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
}

int launch_prompt_tile(const PromptArgs& a, int rows, int src, hipStream_t st);
int launch_prompt_join(const PromptArgs& a, int dtype, hipStream_t st);
int launch_prompt_few(const PromptArgs& a, int dtype, int src, hipStream_t st);

}  // namespace pserve
