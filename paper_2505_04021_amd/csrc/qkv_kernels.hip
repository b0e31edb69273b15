// What lies between a layer's projections and its attention (gfx950): queries and keys are normed head by head and rotated
// to their positions, queries go to a packed tensor, keys and values into the paged cache (the decode step's new token of
// every sequence, or a prefill chunk), in one launch.
//
// Per head x of D elements, in fp32:  y = x * rsqrt(mean x^2 + eps) * w  (where there are weights), then every pair (a, b) of the
// first `rot` elements becomes  m (a cos - b sin),  m (b cos + a sin)  with the angle  position * frequency of the pair.  One
// rounding to bf16 at the end; an e4m3 cache then quantises those bf16 values as kv_append does, so that the cache is what it would
// be had the caller rotated and rounded first.
//
// Angles: position * frequency is off by whole radians in fp32 long before contexts end (2^20 tokens: 2^-4 of a radian), so a
// frequency is held as a fraction of a circle in 64 bits, to the nearest, and multiplied by the position modulo one circle, in integers: within
// 2^-31 of a circle at any position.  v_sin_f32 and v_cos_f32 take that fraction in fp32, 2^-26 of a circle off at most (near half of one); with
// their own error, 2^-22.9 at most over 2^24 fractions of a circle, sine and cosine are 2^-22 off: below what the rounding to bf16 leaves, 2^-8 of an
// outcome, except where a and b all but cancel.
#include "kv_pages.h"

namespace {

// sin and cos of the angle of a pair at a position (any int32: two's complement wraps as the circle does)
__device__ __forceinline__ void turn_of(uint64_t turns, int pos, float &sn, float &cs) {
    const uint32_t lo = (uint32_t)turns, hi = (uint32_t)(turns >> 32);
    const uint32_t at = __umulhi((uint32_t)pos, lo) + (uint32_t)pos * hi - (pos < 0 ? lo : 0u);
    const float rev = (float)(int32_t)at * 0x1p-32f;      // within half a circle either side
    sn = __builtin_amdgcn_sinf(rev);
    cs = __builtin_amdgcn_cosf(rev);
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float bf16_of(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

__device__ __forceinline__ void widen(float *x, const uint32_t *w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = bf16_lo(w[i]);
        x[2 * i + 1] = bf16_hi(w[i]);
    }
}

// The element that e is a pair with.
__device__ __forceinline__ int partner_of(const QkvArgs &a, int e) {
    if (e >= a.rot) return e;
    if (a.pairs) return e ^ 1;
    const int half = a.rot >> 1;
    return e < half ? e + half : e - half;
}

__device__ __forceinline__ float lanes4_sum(float x) {    // over lanes l, l ^ 16, l ^ 32, l ^ 48
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

template <int LANES>
__device__ __forceinline__ float head_sum(float x) {      // over the 8 or 16 lanes that hold a head
    auto add = [&](auto ctrl) __attribute__((always_inline)) {
        x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    add(std::integral_constant<int, 0xb1>{});             // quad_perm: neighbours, then the other pair of the quad
    add(std::integral_constant<int, 0x4e>{});
    add(std::integral_constant<int, 0x141>{});            // mirrored within 8
    if (LANES == 16) add(std::integral_constant<int, 0x140>{});
    return x;
}

__device__ __forceinline__ float square_sum(const uint32_t *w) {
    float x[8], sum = 0.f;
    widen(x, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
    return sum;
}
// (per: 1 / width, a power of two)
__device__ __forceinline__ float norm_of(float squares, float per, float eps) {
#pragma clang fp contract(off)
    return __builtin_amdgcn_rsqf(squares * per + eps);
}

// Keys come by three ways (a lane with two elements of a token's head in a decode step, with groups of eight in a chunk, both of a pair or one of them), and are
// the same to the bit by all of them: what a token leaves in the cache does not depend on the call that brought it.  So every product and sum of
// theirs is written out here, none fused by the compiler, and the squares of a head are summed in one order: by the bits of their places, 6, 5, 0, 1, 2, 3, 4.

// x, p: an element and its partner as they came, w, pw: their weights, r: the head's norm (1 where there is none)
__device__ __forceinline__ float normed_key(float x, float r, float w) {
#pragma clang fp contract(off)
    return (x * r) * w;
}
// an element's outcome from it and its partner, both normed; sn: negative for the first of a pair
__device__ __forceinline__ float turned_key(float x, float p, float sn, float cs) {
#pragma clang fp contract(off)
    return __builtin_fmaf(x, cs, p * sn);
}
// of groups of eight elements, D / 32 of them 32 elements apart: the sum over this lane's; the lanes l, l ^ 16, l ^ 32, l ^ 48 have the others
template <int D>
__device__ __forceinline__ float key_squares(const uint32_t *words) {
#pragma clang fp contract(off)
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float q[D / 32];
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const float x = i & 1 ? bf16_hi(words[4 * j + i / 2]) : bf16_lo(words[4 * j + i / 2]);
            q[j] = x * x;
        }
        if constexpr (D == 128) s[i] = (q[0] + q[2]) + (q[1] + q[3]);
        else s[i] = q[0] + q[1];
    }
    return ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
}
// of elements `lane` and, of 128, lane + 64: the sum over all of the head
__device__ __forceinline__ float key_squares_by_lane(float x0, float x1, bool wide) {
#pragma clang fp contract(off)
    const float a = x0 * x0, b = x1 * x1;
    float s = wide ? a + b : a;
    s = s + __shfl_xor(s, 32);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) s = s + __shfl_xor(s, o);
    return s;
}

// What makes eight elements e0 .. e0 + 7 of a head's outcome at a position: x own + partner other, with the norm's weights and the magnitude in
// it, the same for all heads.  An element that is not rotated has no partner: other = -0, and its partner is taken as 0, so that it stays
// what it is, an infinity and a zero's sign too.
struct Factors {
    float own[8], other[8];
};
__device__ __forceinline__ void eight_weights(float *w, const uint16_t *weight, int e0) {
    const u32x4 v = *reinterpret_cast<const u32x4 *>(weight + e0);
    const uint32_t words[4] = {v.x, v.y, v.z, v.w};
    widen(w, words);
}
// The turns of N pairs in a row (the table has 64 entries, whatever the rotation).
template <int N>
__device__ __forceinline__ void some_turns(uint64_t *t, const QkvArgs &a, int pair) {
    typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const u64x2 v = *reinterpret_cast<const u64x2 *>(a.turns + pair + i);
        t[i] = v.x;
        t[i + 1] = v.y;
    }
}

// The turns of elements e0 .. e0 + 7 (of pairs of neighbours: four) and, but for those, their partners' weights.
template <bool PAIRS>
__device__ __forceinline__ void turns_of_eight(uint64_t *turns, float *pw, const QkvArgs &a, const uint16_t *weight, int e0) {
    const int half = a.rot >> 1;
#pragma unroll
    for (int i = 0; i < 8; ++i) pw[i] = 1.f;
    if constexpr (PAIRS) some_turns<4>(turns, a, e0 >> 1);
    else if ((half & 7) == 0) {                            // a group's partners are a group
        const int low = (e0 < half ? e0 : e0 - half) & 63;
        some_turns<8>(turns, a, low);
        if (weight) eight_weights(pw, weight, partner_of(a, e0));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = e0 + i;
            turns[i] = a.turns[(e < half ? e : e - half) & 63];
            if (weight) pw[i] = bf16_of(weight[partner_of(a, e)]);
        }
    }
}

template <bool PAIRS>
__device__ __forceinline__ Factors factors(const QkvArgs &a, const uint16_t *weight, int e0, int pos, bool rotated) {
    Factors f;
    const int half = a.rot >> 1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f.own[i] = 1.f;
        f.other[i] = -0.f;
    }
    if (weight) eight_weights(f.own, weight, e0);
    if (!rotated) return f;
    uint64_t turns[8];
    float pw[8];
    turns_of_eight<PAIRS>(turns, pw, a, weight, e0);
#pragma unroll
    for (int i = 0; i < 8; i += PAIRS ? 2 : 1) {
        const int e = e0 + i;
        const bool in = e < a.rot;                         // (rot is even: neighbours are rotated or not together)
        float sn, cs;
        turn_of(turns[PAIRS ? i >> 1 : i], pos, sn, cs);
        sn *= a.magnitude;
        cs *= a.magnitude;
        if constexpr (PAIRS) {
            const float o0 = -sn * f.own[i + 1], o1 = sn * f.own[i];
            f.other[i] = in ? o0 : -0.f;
            f.other[i + 1] = in ? o1 : -0.f;
            f.own[i] *= in ? cs : 1.f;
            f.own[i + 1] *= in ? cs : 1.f;
        } else {
            const float o = (e < half ? -sn : sn) * pw[i];
            f.other[i] = in ? o : -0.f;
            f.own[i] *= in ? cs : 1.f;
        }
    }
    return f;
}

// Eight elements' outcome.  xw: their words, pw: their partners' (0 where there is none; not looked at for pairs of neighbours, whose
// partners are among them); r: the head's norm, 1 without one.
template <bool PAIRS>
__device__ __forceinline__ u32x4 turned8(const Factors &f, const uint32_t *xw, const uint32_t *pw, int e0, int rot, float r) {
#pragma clang fp contract(off)
    float x[8], p[8], y[8];
    widen(x, xw);
    if constexpr (PAIRS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = e0 + i < rot ? x[i ^ 1] : 0.f;
    } else widen(p, pw);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_fmaf(x[i] * r, f.own[i], (p[i] * r) * f.other[i]);
    return mk4(pack_bf16_rne(y[0], y[1]), pack_bf16_rne(y[2], y[3]), pack_bf16_rne(y[4], y[5]), pack_bf16_rne(y[6], y[7]));
}

// The eight partners of elements e0 .. e0 + 7 by elements, 0 where there is none.
__device__ __forceinline__ void partners_by_element(const QkvArgs &a, const uint16_t *row, int e0, uint32_t *pw) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = e0 + 2 * i;
        const uint32_t lo = row[partner_of(a, e)], hi = row[partner_of(a, e + 1)];
        pw[i] = (e < a.rot ? lo : 0u) | (e + 1 < a.rot ? hi << 16 : 0u);
    }
}

// The keys of a page on their way into its tile (kv_pages.h).  A lane holds every fourth group of eight elements of its token, so that with half
// layout's partners 32 or 64 elements away it holds both (`near`) and works each angle out once; others are read.  (Factors kept in registers
// for several heads of a page: 237 registers, two waves a SIMD for the queries too.)
template <int D, bool PAIRS>
struct TurnKeys {
    const QkvArgs &a;
    const int pos, c;                                     // this lane's token and column group
    const bool near;
    uint32_t px[D / 32][4];

    __device__ __forceinline__ TurnKeys(const QkvArgs &args, int pos) : a(args), pos(pos), c((int)(threadIdx.x & 63) >> 4), near((args.rot >> 1 & 31) == 0) {}
    __device__ __forceinline__ void ask(const PageRows &p, int t, int) {
        if (PAIRS || near) return;
        int r = t - p.s0;
        r = r < 0 ? 0 : (r < p.n ? r : p.n - 1);
        const uint16_t *row = reinterpret_cast<const uint16_t *>(p.src + (size_t)r * p.stride);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const int e0 = 8 * (4 * j + c);
            if (p.aligned && (a.rot >> 1 & 7) == 0) {
                const u32x4 v = *reinterpret_cast<const u32x4 *>(row + partner_of(a, e0));
#pragma unroll
                for (int i = 0; i < 4; ++i) px[j][i] = e0 < a.rot ? v[i] : 0u;
            } else partners_by_element(a, row, e0, px[j]);
        }
    }
    // groups j and k, pairs 8 (4 j + c) .. + 7: both outcomes
    __device__ __forceinline__ void both(uint32_t *words, int j, int k, float r) {
        const int e0 = 8 * (4 * j + c), e1 = 8 * (4 * k + c);
        float x[8], y[8], wx[8], wy[8];
        widen(x, words + 4 * j);
        widen(y, words + 4 * k);
        uint64_t turns[8];
        some_turns<8>(turns, a, e0);
#pragma unroll
        for (int i = 0; i < 8; ++i) wx[i] = wy[i] = 1.f;
        if (a.k_weight) {
            eight_weights(wx, a.k_weight, e0);
            eight_weights(wy, a.k_weight, e1);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float sn, cs;
            turn_of(turns[i], pos, sn, cs);
            const float p = normed_key(x[i], r, wx[i]), q = normed_key(y[i], r, wy[i]);
            sn *= a.magnitude;
            cs *= a.magnitude;
            x[i] = turned_key(p, q, -sn, cs);
            y[i] = turned_key(q, p, sn, cs);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            words[4 * j + i] = pack_bf16_rne(x[2 * i], x[2 * i + 1]);
            words[4 * k + i] = pack_bf16_rne(y[2 * i], y[2 * i + 1]);
        }
    }
    // group j by itself
    __device__ __forceinline__ void group(uint32_t *words, int j, float r, bool rotated) {
        const int e0 = 8 * (4 * j + c), half = a.rot >> 1;
        float x[8], w[8];
        widen(x, words + 4 * j);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.f;
        if (a.k_weight) eight_weights(w, a.k_weight, e0);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = normed_key(x[i], r, w[i]);
        if (rotated) {
            uint64_t turns[8];
            float p[8], pw[8];
            turns_of_eight<PAIRS>(turns, pw, a, a.k_weight, e0);
            if constexpr (!PAIRS) widen(p, px[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = PAIRS ? x[i ^ 1] : normed_key(p[i], r, pw[i]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = e0 + i;
                float sn, cs;
                turn_of(turns[PAIRS ? i >> 1 : i], pos, sn, cs);
                sn *= a.magnitude;
                cs *= a.magnitude;
                const float y = turned_key(x[i], p[i], (PAIRS ? (i & 1) == 0 : e < half) ? -sn : sn, cs);
                x[i] = e < a.rot ? y : x[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) words[4 * j + i] = pack_bf16_rne(x[2 * i], x[2 * i + 1]);
    }
    __device__ __forceinline__ void turn(uint32_t *words) {
        if (!a.turns && !a.k_weight) return;
        float r = 1.f;
        if (a.k_weight) r = norm_of(lanes4_sum(key_squares<D>(words)), 1.f / D, a.eps);
        if (!PAIRS && a.turns && near) {
            if (D == 128 && a.rot == 128) {
                both(words, 0, D == 128 ? 2 : 1, r);
                both(words, 1, D == 128 ? 3 : 1, r);
            } else {                                       // rot = 64
                both(words, 0, 1, r);
                if (D == 128 && a.k_weight) {
#pragma unroll
                    for (int j = 2; j < D / 32; ++j) group(words, j, r, false);
                }
            }
            return;
        }
        // (a condition for the whole wave: lanes of one group of eight differ in it only where rot is no multiple of 32)
#pragma unroll
        for (int j = 0; j < D / 32; ++j) group(words, j, r, a.turns && 32 * j < a.rot);
    }
};

// Heads head0 .. head0 + heads - 1 of one token's query, 8 elements a lane, 512 / D heads at a time: whole rows of 16-byte pieces.  The
// first rows are asked for ahead of the token's position (pos_of()), the next ones ahead of the arithmetic of those before.
template <int D, bool PAIRS, typename POS_OF>
__device__ __forceinline__ void turn_queries(const AttnDesc &d, const QkvArgs &a, int64_t row, int head0, int heads, const POS_OF &pos_of) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES, BATCH = 4;
    const int lane = threadIdx.x & 63, c = lane % LANES, e0 = 8 * c, half = a.rot >> 1;
    const uint16_t *src = a.q + row * a.q_stride;
    uint16_t *dst = a.q_out + row * d.Hq * D;
    auto head_of = [&](int h0) __attribute__((always_inline)) { return h0 + lane / LANES; };
    auto load = [&](u32x4 *x, int h0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int h = head_of(h0 + k * ROWS);
            const uint16_t *at = src + (h < head0 + heads ? h : head0) * D + e0;
            if (a.q_aligned) x[k] = *reinterpret_cast<const u32x4 *>(at);
            else x[k] = mk4(at[0] | (uint32_t)at[1] << 16, at[2] | (uint32_t)at[3] << 16, at[4] | (uint32_t)at[5] << 16, at[6] | (uint32_t)at[7] << 16);
        }
        asked_for();
    };
    u32x4 x[BATCH], next[BATCH];
    load(x, head0);
    const Factors f = factors<PAIRS>(a, a.q_weight, e0, pos_of(), a.turns != nullptr);
    const bool whole = (half & 7) == 0;                   // a group's partners are a group
    const int from = lane - c + (!PAIRS && whole ? partner_of(a, e0) >> 3 : c);
    for (int h0 = head0; h0 < head0 + heads; h0 += BATCH * ROWS) {
        const bool more = h0 + BATCH * ROWS < head0 + heads;
        if (more) load(next, h0 + BATCH * ROWS);
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            if (h0 + k * ROWS >= head0 + heads) break;
            const int h = head_of(h0 + k * ROWS);
            const bool live = h < head0 + heads;
            uint32_t xw[4], pw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                xw[i] = x[k][i];
                pw[i] = 0u;
            }
            if (!PAIRS && a.turns) {
                if (whole) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t w = (uint32_t)__shfl((int)xw[i], from);
                        pw[i] = e0 < a.rot ? w : 0u;
                    }
                } else partners_by_element(a, src + (live ? h : head0) * D, e0, pw);
            }
            const float r = a.q_weight ? norm_of(head_sum<LANES>(square_sum(xw)), 1.f / D, a.eps) : 1.f;
            const u32x4 y = turned8<PAIRS>(f, xw, pw, e0, a.rot, r);
            if (live) *reinterpret_cast<u32x4 *>(dst + h * D + e0) = y;
        }
        if (more) {
#pragma unroll
            for (int k = 0; k < BATCH; ++k) x[k] = next[k];
        }
    }
}

template <typename POS_OF>
__device__ __forceinline__ void turn_queries(const AttnDesc &d, const QkvArgs &a, int64_t row, int head0, const POS_OF &pos_of) {
    const int heads = d.Hq - head0 < a.wave_heads ? d.Hq - head0 : a.wave_heads;
    if (d.D == 128) {
        if (a.pairs) turn_queries<128, true>(d, a, row, head0, heads, pos_of);
        else turn_queries<128, false>(d, a, row, head0, heads, pos_of);
    } else {
        if (a.pairs) turn_queries<64, true>(d, a, row, head0, heads, pos_of);
        else turn_queries<64, false>(d, a, row, head0, heads, pos_of);
    }
}

// The decode step.  One wave per (sequence, kv head) for K and V of its new token, the element layout of k_kv_append, then
// waves for the queries.  Bound by dependent memory trips (context length, block id, the block): 64 rows of 32/8/128 4.0 us, into an e4m3 cache
// 5.3, and 19.9 where every token raises its blocks' scales (the codes of earlier slots go one slot after the other).
template <int DT>
__global__ __launch_bounds__(64) void k_qkv_append(const AttnDesc d, const QkvArgs a) {
    const int lane = threadIdx.x, D = d.D, kv_waves = d.batch * d.Hkv;
    if ((int)blockIdx.x >= kv_waves) {
        const int x = blockIdx.x - kv_waves, per = (d.Hq + a.wave_heads - 1) / a.wave_heads, seq = x / per;
        turn_queries(d, a, seq, (x - seq * per) * a.wave_heads, [&]() __attribute__((always_inline)) {
            return (a.before ? PKV_CONST(int32_t, a.before)[seq] : 0) + PKV_CONST(int32_t, d.ctx_lens)[seq] - 1;
        });
        return;
    }
    const int seq = blockIdx.x / d.Hkv, h = blockIdx.x - seq * d.Hkv;
    const uint16_t *k = a.k + seq * a.k_stride + (size_t)h * D, *v = a.v + seq * a.v_stride + (size_t)h * D;
    const int second = lane + (D > 64 ? 64 : 0);
    uint32_t kx[2] = {k[lane], k[second]}, vx[2] = {v[lane], v[second]}, kp[2] = {k[partner_of(a, lane)], k[partner_of(a, second)]};
    const int ctx = PKV_CONST(int32_t, d.ctx_lens)[seq], before = a.before ? PKV_CONST(int32_t, a.before)[seq] : 0;
    const int cap = PKV_CONST(int32_t, d.row_len)[seq] * PKV_T;
    if ((ctx < 1) | (ctx > cap)) {
        if (lane == 0) atomicOr(d.err, 2u);
        return;
    }
    const uint32_t id = (uint32_t)PKV_CONST(int32_t, d.table)[(size_t)seq * d.row_stride + (ctx - 1) / PKV_T];
    if (id >= d.max_block_id) {
        if (lane == 0) atomicOr(d.err, 1u);
        return;
    }
    if (a.turns || a.k_weight) {
        float x[2] = {bf16_lo(kx[0]), bf16_lo(kx[1])}, p[2] = {bf16_lo(kp[0]), bf16_lo(kp[1])};
        float r = 1.f;
        if (a.k_weight) r = norm_of(key_squares_by_lane(x[0], x[1], D > 64), D > 64 ? 1.f / 128 : 1.f / 64, a.eps);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = i ? second : lane, pe = partner_of(a, e), half = a.rot >> 1;
            if (a.k_weight) {
                x[i] = normed_key(x[i], r, bf16_of(a.k_weight[e]));
                p[i] = normed_key(p[i], r, bf16_of(a.k_weight[pe]));
            }
            if (a.turns && e < a.rot) {
                const int pair = a.pairs ? e >> 1 : (e < half ? e : e - half);
                float s, c;
                turn_of(a.turns[pair], before + ctx - 1, s, c);
                s *= a.magnitude;
                x[i] = turned_key(x[i], p[i], e < pe ? -s : s, c * a.magnitude);
            }
            kx[i] = pack_bf16_rne(x[i], 0.f) & 0xffffu;
        }
    }
    uint8_t *blk = block_ptr(d, id);
    const int slot = (ctx - 1) % PKV_T;
    if (DT == PKV_BF16) {
        const size_t tile = (size_t)PKV_T * D * 2;
        uint16_t *kt = reinterpret_cast<uint16_t *>(blk + (size_t)h * 2 * tile);
        uint16_t *vt = reinterpret_cast<uint16_t *>(blk + (size_t)h * 2 * tile + tile);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int dd = lane + 64 * i;
            if (dd < D) {
                kt[k_elem_off<PKV_BF16>(slot, dd)] = (uint16_t)kx[i];
                vt[v_elem_off<PKV_BF16>(slot, dd)] = (uint16_t)vx[i];
            }
        }
    } else {
        float *hdr = reinterpret_cast<float *>(blk);
        const size_t tile = (size_t)PKV_T * D;
        uint8_t *kt = blk + PKV_FP8_HEADER + (size_t)h * 2 * tile, *vt = kt + tile;
        if (D == 64) kx[1] = vx[1] = 0u;
        append_row_e4m3<false>(kt, hdr + h, slot, D, kx, lane);
        append_row_e4m3<true>(vt, hdr + d.Hkv + h, slot, D, vx, lane);
    }
}

// Bound by memory: ragged prompts of 4300 tokens of 32/8/128, neighbours as pairs, 115 MB, cold: 26.1 us (22.6 at a large copy's rate).  39.0 with every head's weights and angles looked up and worked out by themselves, one row in flight a wave;
// 96 registers, five waves a SIMD; with 80, six, some 200 to 350 spill (bf16 26.0, e4m3 with its way back 23.9 instead of 19.5).
// 2400 tokens into an e4m3 cache 15.9 (first kernel 23.5), 4.9 million vector instructions, some 9 us of issue, beside 46 MB.
// With V read in pieces of 8 bytes 26.5.
// A prefill chunk.  Waves of whole pages as in k_kv_append_chunk (one per page that the chunk touches, kv head, and K or V), then waves for
// the queries, each with some heads of one token.  (Queries first: the prompts above 29.6 us, 27.5 so; 2000 tokens into an e4m3 cache, with their way
// back, 21.0, 19.6.)
constexpr int QKV_WAVES = 4;

// How many drafted tokens, of its sequence's n, are in front of one on its path.
__device__ __forceinline__ int depth_of(const uint64_t *row, int words, int n) {
    const int seen = seen_drafts(row, words, n);
    return seen > 0 ? seen - 1 : 0;
}

// TREE: drafted tokens, whose positions go by how many drafted tokens each sees (its row of a.sees).  714 of 32/8/128, 18 MB: 9.4 us, two thirds of the waves' time
// waiting for dependent trips (the same tokens as a chunk 10.4).
template <int D, int DT, int SEQS, bool TREE>
__global__ __launch_bounds__(64 * QKV_WAVES, 4) void k_qkv_append_chunk(const AttnDesc d, const QkvArgs a, const PlanOf<SEQS> plan) {
    constexpr int E = DT == PKV_BF16 ? 2 : 1;
    const int lane = threadIdx.x & 63;
    const PlanLanes<SEQS> lanes(plan);
    const int n_seqs = plan.n_seqs;
    int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * QKV_WAVES + (threadIdx.x >> 6)));
    const int page_waves = (int)lanes.units(plan) * d.Hkv * 2;
    if (x >= page_waves) {
        x -= page_waves;
        const int per = (d.Hq + a.wave_heads - 1) / a.wave_heads, row0 = (int)(lanes.pick(lanes.row, 0) & PKV_PLAN_ROWS);
        const int row = row0 + x / per;
        if (row >= (int)(lanes.pick(lanes.row, n_seqs) & PKV_PLAN_ROWS)) return;           // the last work-group may have waves to spare
        turn_queries(d, a, row, (x % per) * a.wave_heads, [&]() __attribute__((always_inline)) {
            const PlanUnit pu = lanes.find_row(plan, (uint32_t)row);
            if constexpr (TREE)
                return (a.before ? PKV_CONST(int32_t, a.before)[pu.seq] : 0) + PKV_CONST(int32_t, d.ctx_lens)[pu.seq] - pu.rows +
                       depth_of(a.sees + (size_t)row * a.words, a.words, pu.rows);
            return (a.before ? PKV_CONST(int32_t, a.before)[pu.seq] : 0) + PKV_CONST(int32_t, d.ctx_lens)[pu.seq] - pu.rows + row - pu.row;
        });
        return;
    }
    const bool keys = (x & 1) == 0;
    const int unit = (x >> 1) / d.Hkv, h = (x >> 1) - unit * d.Hkv;
    const PlanUnit pu = lanes.find(plan, (uint32_t)unit);
    const int ctx = PKV_CONST(int32_t, d.ctx_lens)[pu.seq], cap = PKV_CONST(int32_t, d.row_len)[pu.seq] * PKV_T;
    if ((ctx < pu.rows) | (ctx < 1) | (ctx > cap)) {
        if (lane == 0) atomicOr(d.err, 2u);
        return;
    }
    const int tok0 = ctx - pu.rows, page = tok0 / PKV_T + pu.unit;
    const int lo = tok0 > page * PKV_T ? tok0 : page * PKV_T, hi = ctx < (page + 1) * PKV_T ? ctx : (page + 1) * PKV_T;
    if (lo >= hi) return;
    const uint32_t id = (uint32_t)PKV_CONST(int32_t, d.table)[(size_t)pu.seq * d.row_stride + page];
    const uint16_t *src = keys ? a.k : a.v;
    const int64_t stride = keys ? a.k_stride : a.v_stride;
    PageRows p;
    p.stride = (size_t)stride * 2;
    p.s0 = lo % PKV_T;
    p.n = hi - lo;
    p.aligned = ((reinterpret_cast<uintptr_t>(src) | (uintptr_t)(stride * 2)) & 15) == 0;
    p.src = reinterpret_cast<const uint8_t *>(src + (pu.row + (lo - tok0)) * stride + (size_t)h * D);
    auto page_of = [&](auto is_v, auto &&turn) __attribute__((always_inline)) {
        constexpr bool IS_V = decltype(is_v)::value;
        auto block = [&]() __attribute__((always_inline)) -> uint8_t * {
            if (id >= d.max_block_id) {
                if (lane == 0) atomicOr(d.err, 1u);
                return nullptr;
            }
            return block_ptr(d, id);
        };
        const size_t offset = (DT == PKV_E4M3 ? PKV_FP8_HEADER : 0) + ((size_t)h * 2 + (IS_V ? 1 : 0)) * PKV_T * D * E;
        if constexpr (DT == PKV_BF16) {
            page_bf16<D, IS_V>([&]() __attribute__((always_inline)) -> uint8_t * {
                uint8_t *blk = block();
                return blk ? blk + offset : blk;
            }, p, turn);
        } else {
            page_quantise<D, IS_V>([&](float *&scale_p) __attribute__((always_inline)) -> uint8_t * {
                uint8_t *blk = block();
                scale_p = reinterpret_cast<float *>(blk) + (IS_V ? d.Hkv : 0) + h;
                return blk ? blk + offset : blk;
            }, p, turn);
        }
    };
    if (!keys) {
        page_of(std::true_type{}, AsTheyAre{});
        return;
    }
    int pos = (a.before ? PKV_CONST(int32_t, a.before)[pu.seq] : 0) + page * PKV_T + (lane & 15);
    if constexpr (TREE) {
        int i = page * PKV_T + (lane & 15) - tok0;         // (a slot that gets no token takes the position of one that does)
        i = i < 0 ? 0 : (i < pu.rows ? i : pu.rows - 1);
        pos = (a.before ? PKV_CONST(int32_t, a.before)[pu.seq] : 0) + tok0 + depth_of(a.sees + (size_t)(pu.row + i) * a.words, a.words, pu.rows);
    }
    if (a.pairs) page_of(std::false_type{}, TurnKeys<D, true>(a, pos));
    else page_of(std::false_type{}, TurnKeys<D, false>(a, pos));
}

}  // namespace

hipError_t pkv_launch_qkv_append(const AttnDesc &d, const QkvArgs &a, hipStream_t s) {
    const unsigned waves = (unsigned)d.batch * (unsigned)(d.Hkv + (d.Hq + a.wave_heads - 1) / a.wave_heads);
    if (waves == 0) return hipSuccess;
    if (d.dtype == PKV_BF16) hipLaunchKernelGGL(k_qkv_append<PKV_BF16>, dim3(waves), dim3(64), 0, s, d, a);
    else hipLaunchKernelGGL(k_qkv_append<PKV_E4M3>, dim3(waves), dim3(64), 0, s, d, a);
    return hipGetLastError();
}

template <int SEQS, bool TREE>
static void launch_chunk(const AttnDesc &d, const QkvArgs &a, const PlanOf<SEQS> &plan, dim3 grid, hipStream_t s) {
    static_assert(sizeof(AttnDesc) + sizeof(QkvArgs) + sizeof(PlanOf<SEQS>) <= 4096, "a kernel's arguments end at 4 KB");
    const dim3 wg(64 * QKV_WAVES);
    if (d.dtype == PKV_BF16) {
        if (d.D == 128) hipLaunchKernelGGL((k_qkv_append_chunk<128, PKV_BF16, SEQS, TREE>), grid, wg, 0, s, d, a, plan);
        else hipLaunchKernelGGL((k_qkv_append_chunk<64, PKV_BF16, SEQS, TREE>), grid, wg, 0, s, d, a, plan);
    } else {
        if (d.D == 128) hipLaunchKernelGGL((k_qkv_append_chunk<128, PKV_E4M3, SEQS, TREE>), grid, wg, 0, s, d, a, plan);
        else hipLaunchKernelGGL((k_qkv_append_chunk<64, PKV_E4M3, SEQS, TREE>), grid, wg, 0, s, d, a, plan);
    }
}

hipError_t pkv_launch_qkv_append_chunk(const AttnDesc &d, const QkvArgs &a, const ChunkPlan &plan, hipStream_t s) {
    const uint64_t rows = (plan.s[plan.n_seqs].row & PKV_PLAN_ROWS) - (plan.s[0].row & PKV_PLAN_ROWS), units = plan.s[plan.n_seqs].unit;
    const uint64_t waves = units * (uint64_t)d.Hkv * 2 + rows * (uint64_t)((d.Hq + a.wave_heads - 1) / a.wave_heads);
    if (rows == 0) return hipSuccess;
    if (waves > 0x7fffffffu) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)((waves + QKV_WAVES - 1) / QKV_WAVES));
    if (plan.n_seqs <= PKV_PLAN_FEW) {
        if (a.sees) launch_chunk<PKV_PLAN_FEW, true>(d, a, few_of(plan), grid, s);
        else launch_chunk<PKV_PLAN_FEW, false>(d, a, few_of(plan), grid, s);
    } else {
        if (a.sees) launch_chunk<PKV_PLAN_SEQS, true>(d, a, plan, grid, s);
        else launch_chunk<PKV_PLAN_SEQS, false>(d, a, plan, grid, s);
    }
    return hipGetLastError();
}
