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
    int32_t n, Hk, G, D, causal;
    int32_t rows, splits;               // rows of a tile, shares of its keys (wide tiles)
    int32_t unit, lead, blocks;         // tiles of 16 rows: keys of a unit of work (0: tiles are not cut), units a tile costs besides, blocks
    int32_t items;                      // tiles that are not cut: slots of tiles times key/value heads
    int32_t max_pages, page_shift;
    uint32_t pages, places;             // SRC_STORE: of the store; the last page may be filled in part
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
// The i-th tile of R rows in the order that the blocks take them, over sequences of cu_q[s + 1] - cu_q[s] tokens of G rows each, without a
// table made by the host.  There are at most `slots` = prompt_slots of them; false: i has none.
// Of a sequence the last tile comes first (under a causal mask it has the most keys).  Up to 64 sequences, one a lane, are numbered without
// gaps, so the blocks that have no tile are the last; more have the slots from floor(cu_q[s] G / R) + s on, at least as many as they
// have tiles, found by a search.  Where the keys are cut into shares the sequences with the most keys come first, so that no long tile is left
// for the end (4 of 77 .. 640 tokens over 717 .. 4095 stored keys, the longest in front: 78 -> 71 us, heads of 128 110 -> 80); else the
// last sequence does, as ordering them takes 2 us of every block's time with 32 sequences (32 prompts of 512: 249 us without, 265 with).
// (Gaps cost a round of blocks where the tiles just fill the chip, as blocks are dealt out in a fixed order: 32 sequences of 8 tokens over 2000
// keys, 2 tiles and a gap each, 62 us with gaps, 45 without; 32 prompts of 77 with 12 heads 15 and 11; 32 of 512, where the gaps moved
// long tiles against each other, 240 and 249.  A walk over all of 16,384 sequences in every block takes 66 ms where the search takes 2.)
template <int SRC>
__device__ __forceinline__ bool prompt_slot(const PromptArgs& a, int G, int R, int64_t slots, int64_t i, int& s, int& tile) {
    const int lane = threadIdx.x & 63;
    if (a.n <= 64) {
        PromptSeq q{0, 0, 0, 0};
        if (lane < a.n) q = prompt_seq<SRC>(a, lane);
        const int tiles = (int)(((int64_t)q.Lq * G + R - 1) / R);
        int before = 0;                         // tiles of the sequences in front
        if (a.splits > 1) {
            for (int j = 0; j < a.n; ++j) {
                const int kj = __builtin_amdgcn_readlane(q.Lk, j), tj = __builtin_amdgcn_readlane(tiles, j);
                if (kj > q.Lk || (kj == q.Lk && j > lane)) before += tj;
            }
        } else {
            int upto = tiles;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(upto, d);
                if (lane >= d) upto += o;
            }
            before = __builtin_amdgcn_readlane(upto, 63) - upto;
        }
        const uint64_t at = __ballot(i >= before && i < (int64_t)before + tiles);
        if (at == 0) return false;
        s = __ffsll((unsigned long long)at) - 1;
        tile = __builtin_amdgcn_readlane(before, s) + __builtin_amdgcn_readlane(tiles, s) - 1 - (int)i;
        return true;
    }
    // the last sequence whose slots begin at `slot` or in front of it, 64 places of the range looked at in one go; where the starts do
    // not ascend, any one
    const int64_t slot = slots - 1 - i;
    int lo = 0, len = a.n;
    for (;;) {
        const int step = (len + 63) / 64, at = lo + lane * step;
        const bool le = lane * step < len && prompt_start(a.cu_q, at, a.q_tokens) * G / R + at <= slot;
        const uint64_t past = ~__ballot(le);
        const int count = past ? __ffsll((unsigned long long)past) - 1 : 64;
        if (count == 0) return false;
        lo += (count - 1) * step;
        len = min(step, len - (count - 1) * step);
        if (step == 1) break;
    }
    s = __builtin_amdgcn_readfirstlane(lo);
    tile = (int)(slot - (prompt_start(a.cu_q, s, a.q_tokens) * G / R + s));
    return true;
}
// SRC_STORE: the place of a sequence's key, -1: none of the store's.  A page of the store starts below `places` <= 2^31 - 1, and has at most 2^30
__device__ __forceinline__ int prompt_place(const PromptArgs& a, int s, int key) {
    const uint32_t page = (uint32_t)a.table[(int64_t)s * a.max_pages + (key >> a.page_shift)];
    const uint32_t place = page << a.page_shift | ((uint32_t)key & ((1u << a.page_shift) - 1));
    return page < a.pages && place < a.places ? (int)place : -1;
}
inline int64_t prompt_slots(const PromptArgs& a, int G, int R) { return a.q_tokens * G / R + a.n; }

// The work of the 16-row tiles, where they are cut, in units of `unit` keys of one tile: sequence s has tiles x Hk x U_s of them, the blocks
// take equal runs of the numbered units, whatever the sequences' lengths are.  The first `lead` units of a tile stand for what it costs besides its keys (its
// queries, the way to the first keys, the meeting of the wavefronts): without them a block of short sequences is the last to end.  Every
// wavefront walks the sequences by itself, 64 at a time, one a lane (tiles are cut where there are fewer than 768).
__device__ __forceinline__ int64_t uniform64(int64_t v) {      // the same in all lanes: into scalar registers
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ int64_t lane64(int64_t v, int l) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, l));
}
template <int SRC>
struct PromptWalk {
    const PromptArgs& a;
    int first = 0;                      // sequence of lane 0
    int64_t before = 0;                 // units of the sequences in front of it
    PromptSeq q;                        // the lane's sequence
    int U = 1;                          // units of one of its tiles
    int64_t units = 0, upto = 0;        // its units; those from `first` up to its end
    // of the unit found: sequence and the number of its first unit
    int s = 0;
    int64_t base = 0;

    __device__ __forceinline__ explicit PromptWalk(const PromptArgs& a_) : a(a_) {
        if (a.unit) load();
    }
    __device__ __forceinline__ void load() {
        const int lane = threadIdx.x & 63;
        units = 0;
        if (first + lane < a.n) {
            q = prompt_seq<SRC>(a, first + lane);
            U = max(1, (int)(((int64_t)q.Lk + a.unit - 1) / a.unit)) + a.lead;
            units = ((int64_t)q.Lq * a.G + 15) / 16 * a.Hk * U;
        }
        upto = units;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
    }
    __device__ __forceinline__ int64_t total() {                // units of all sequences; the walk starts over
        int64_t sum = lane64(upto, 63);
        if (a.n > 64) {
            for (first = 64; first < a.n; first += 64) {
                load();
                sum += lane64(upto, 63);
            }
            first = 0;
            load();
        }
        return sum;
    }
    // the sequence that holds unit w, which lies behind the unit found before; false: none
    __device__ __forceinline__ bool find(int64_t w) {
        for (;;) {
            const uint64_t past = __ballot(before + upto > w);
            if (past) {
                const int l = __ffsll((unsigned long long)past) - 1;
                s = first + l;
                base = before + lane64(upto, l) - lane64(units, l);
                return true;
            }
            if (first + 64 >= a.n) return false;
            before += lane64(upto, 63);
            first += 64;
            load();
        }
    }
    __device__ __forceinline__ PromptSeq seq() const {
        const int l = s - first;
        PromptSeq r;
        r.q0 = lane64(q.q0, l);
        r.k0 = lane64(q.k0, l);
        r.Lq = __builtin_amdgcn_readlane(q.Lq, l);
        r.Lk = __builtin_amdgcn_readlane(q.Lk, l);
        return r;
    }
    __device__ __forceinline__ int tile_units() const { return __builtin_amdgcn_readlane(U, s - first); }
};
// W units over the blocks: block b has those from floor(W b / B) on.  No more blocks than units have any.  (A 64-bit division takes a
// hundred instructions: there is one here, and none where every block has one unit.)
struct PromptShares {
    int64_t W, B, whole;
    uint32_t rest;
    __device__ __forceinline__ PromptShares(const PromptArgs& a, int64_t W_) : W(W_), B(min((int64_t)a.blocks, W_)) {
        whole = 1;
        rest = 0;
        if (W > B) {
            whole = W / B;
            rest = (uint32_t)(W - whole * B);
        }
    }
    __device__ __forceinline__ int64_t begin(int64_t b) const {
        return whole * b + (rest == 0 ? 0 : B <= 65536 ? (int64_t)(rest * (uint32_t)b / (uint32_t)B) : (int64_t)rest * b / B);
    }
    __device__ __forceinline__ int64_t block_of(int64_t w) const {
        int64_t b = (int64_t)((double)w * (double)B / (double)W);
        while (begin(b + 1) <= w) ++b;
        while (begin(b) > w) --b;
        return b;
    }
};
// quotient and rest of a run of units by the units of a tile
__device__ __forceinline__ int prompt_item(int64_t units, int U, int& off) {
    if (units >> 32 == 0) {
        const uint32_t i = (uint32_t)units / (uint32_t)U;
        off = (int)((uint32_t)units - i * (uint32_t)U);
        return (int)i;
    }
    off = (int)(units % U);
    return (int)(units / U);
}

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;

// two whole numbers of a dword of four (bytes 2 h, 2 h + 1) as a pair of bf16: exact, 7 bits and a sign
__device__ __forceinline__ uint32_t bf16_of_i8(uint32_t w, int h) {
    const float lo = (float)(int8_t)(w >> (16 * h)), hi = (float)(int8_t)(w >> (16 * h + 8));
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
}

int launch_prompt_tile(const PromptArgs& a, int rows, int src, hipStream_t st);
int launch_prompt_join(const PromptArgs& a, int src, hipStream_t st);
int launch_prompt_few(const PromptArgs& a, int dtype, int src, hipStream_t st);

}  // namespace pserve
