// Which tokens a query sees where that is not simply "all up to its own" (gfx950): a sliding window with sinks, or the ancestors of a
// drafted token behind its context.
//
//   out = softmax over the seen t of (q . k_t / sqrt D) V
//
// A query at position p sees token t <= p where t > p - window or t < sinks.  A drafted token sees the cached tokens in front of the drafts by the
// same rule, p being the position that its depth gives it, and of the drafted ones those whose bit is set in its row of the mask.
#pragma once
#include "mfma_util.h"

namespace {

// bits 0 .. n - 1
__device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? 0xffffffffu : (n <= 0 ? 0u : (1u << n) - 1u); }

// A column's 32 tokens from x0 on: seen are those below `hi` that are sinks or not below `lo`
__device__ __forceinline__ uint32_t seen_bits(int x0, int hi, int lo, int sinks) {
    return below(hi - x0) & (~below(lo - x0) | below(sinks - x0));
}

// The tokens that some query of a unit may see, as one walk along pages: the sinks' pages, then those from the first query's window on.
// Tokens are counted along the walk: those behind the gap are 16 * skip fewer than in the row.
struct Walk {
    int len;                 // tokens, to the end of what the last query sees
    int front, skip;         // pages in front of the gap; pages left out
    int sinks;               // tokens in front that every query sees
    int lo_min, lo_max;      // where the windows of the first and of the last query begin
    int hi_min;              // tokens that all queries see, but for the windows
    __device__ __forceinline__ int page(int i) const { return i < front ? i : i + skip; }
    __device__ __forceinline__ int pages() const { return (len + PKV_T - 1) / PKV_T; }
    // of the 32 tokens from x0 on those that some query sees, as bits
    __device__ __forceinline__ uint32_t some(int x0) const { return seen_bits(x0, len, lo_min, sinks); }
    // whether every query sees all 32 tokens from x0 on
    __device__ __forceinline__ bool plain(int x0) const { return (x0 + 32 <= hi_min) & ((x0 >= lo_max) | (x0 + 32 <= sinks)); }
};

// L tokens of the row; windows that begin at token `lo_min` and `lo_max`; all queries see tokens below `hi_min`, as far as windows go
__device__ __forceinline__ Walk walk_of(int L, int lo_min, int lo_max, int hi_min, int sinks) {
    Walk w;
    L = L < 0 ? 0 : L;
    auto within = [&](int x) __attribute__((always_inline)) { return x < 0 ? 0 : (x < L ? x : L); };
    w.sinks = within(sinks);
    lo_min = within(lo_min);
    w.front = (w.sinks + PKV_T - 1) / PKV_T;
    const int first = lo_min / PKV_T;
    w.skip = first > w.front ? first - w.front : 0;
    const int shift = w.skip * PKV_T;
    w.len = L - shift;
    w.lo_min = lo_min - shift;
    w.lo_max = within(lo_max) - shift;
    w.hi_min = within(hi_min) - shift;
    return w;
}

// Rows of a tree's mask in LDS: bits [from, from + 32) of a row of `words` 32-bit words, zeros beyond it
__device__ __forceinline__ uint32_t row_bits(const uint32_t *row, int words, int from) {
    const int i = from >> 5;                              // (arithmetic: -1 for the 32 bits in front)
    auto word = [&](int k) __attribute__((always_inline)) {
        const uint32_t x = row[k < 0 ? 0 : (k < words ? k : words - 1)];
        return k >= 0 && k < words ? x : 0u;
    };
    return __builtin_amdgcn_alignbit(word(i + 1), word(i), (uint32_t)from & 31u);
}

// Two bits as masks of two 16-bit values, four bits as masks of four bytes.
__device__ __forceinline__ uint32_t halves_of(uint32_t two) { return (two & 1u ? 0xffffu : 0u) | (two & 2u ? 0xffff0000u : 0u); }
__device__ __forceinline__ uint32_t bytes_of(uint32_t four) {
    return (four & 1u ? 0xffu : 0u) | (four & 2u ? 0xff00u : 0u) | (four & 4u ? 0xff0000u : 0u) | (four & 8u ? 0xff000000u : 0u);
}

// Infinities and NaN in V.  A token that some columns of a tile see and others do not has the probability 0 in the others' products, and 0 * NaN spoils their sums.
// So a wave whose sums are not all finite at its walk's end walks once more, with zeros for what is not finite in V; what sees such an element is
// spoiled by finite factors: products of 2^127 where the element is not finite with +-2^127 where the column sees the token are infinities of both signs, and 0
// elsewhere.  (Looking through V in every pair under masks, and this in the walk itself, took 1 to 10 % of all calls' time, and registers that there are not.)
__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
// the halves of a word of bf16 values that are no finite ones, as masks
__device__ __forceinline__ uint32_t strange_halves(uint32_t w) {
    return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}
// a word of V with zeros for what is not finite
template <int DT>
__device__ __forceinline__ uint32_t finite_only(uint32_t w) {
    if constexpr (DT == PKV_BF16) return w & ~strange_halves(w);
    else return w & ~((((w & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xffu);
}
constexpr uint32_t kSpoil = 0x7f007f00u, kMinusSpoil = 0xff00ff00u;  // two bf16 values, 2^127 and its negative

constexpr int MASK_WORDS = 2 * PKV_TREE_WORDS;           // 32-bit words of a row of a tree's mask in LDS

}  // namespace
