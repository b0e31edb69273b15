// Attention under masks (mask_walk.h): the work-group that walks one part of a context for up to 16 or 32 columns (gfx950).
#pragma once
#include "decode_part.h"
#include "mask_walk.h"

namespace {

// One work-group's part of a launch: its columns are `tokens` query tokens x the g heads of a kv head.
struct MaskUnit {
    int seq, kvh, part, parts, size;     // which of how many parts of the walk, of how many pages
    int first, tokens;                   // rows of q and out
    int slot;                            // arrival counter of the unit
    size_t partial;                      // its partial sums (of part 0; the others follow `step` apart)
    size_t step;
    int chunk0, chunk;                   // the first of them among its sequence's, and how many those are
};

// Blanks the tokens of a V tile that no query sees, which may hold anything (even NaN); a set bit: seen
template <int D, int DT>
__device__ __forceinline__ void keep_v(u32x4 *v, uint32_t four) {
    const uint32_t m01 = halves_of(four), m23 = halves_of(four >> 2), m = bytes_of(four);
#pragma unroll
    for (int j = 0; j < Tile<D, DT>::NL; ++j) v[j] &= DT == PKV_BF16 ? mk4(m01, m23, m01, m23) : mk4(m, m, m, m);
}

// Columns of a unit: one or two tiles of 16.
template <int NT>
constexpr int kMaskCols = 16 * NT;
// LDS of a work-group: the sums of its four waves, or what the last one to arrive reads of all parts.
template <int NT>
constexpr int kMaskSums = SMALL_WAVES * 16 * NT * 128;
static_assert(kMaskSums<1> >= 2 * MAX_PIECES * 16 && kMaskSums<2> >= 2 * MAX_PIECES * 32, "room for the maxima and denominators of all parts");

// The work-group's four waves take the page pairs of its part in turn and join their sums through LDS; the last of several parts to arrive joins
// those through memory (as attn_part in decode_part.h, whose comments say why it is built like this).
// With two tiles of columns a wave keeps one pair: K of the next pair is asked for when the scores have been taken, V when the products have, in the
// registers that have become free.
template <int D, int DT, int NT, bool TREE>
__device__ __forceinline__ void masked_part(const AttnDesc &d, const MaskArgs &mk, const MaskUnit &u, float *s_acc, float *s_m, float *s_l, uint32_t *s_mask,
                                            uint32_t *s_arrived) {
    using TL = Tile<D, DT>;
    constexpr int MC = kMaskCols<NT>;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int G = lane >> 4, n = lane & 15, g = d.g, cols = u.tokens * g;
    const int32_t *row = d.table + (size_t)u.seq * d.row_stride;
    bf16x8 qf[NT][TL::NK];
    int tok[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        const int col = 16 * c + n;
        const bool live = col < cols;
        tok[c] = live ? col / g : 0;
        const uint16_t *qrow = d.q + ((size_t)(u.first + tok[c]) * d.Hq + u.kvh * g + (live ? col - tok[c] * g : 0)) * D;
#pragma unroll
        for (int j = 0; j < TL::NK; ++j) {
            u32x4 v = mk4(0, 0, 0, 0);
            if (live) v = *reinterpret_cast<const u32x4 *>(qrow + 8 * (4 * j + G));
            qf[c][j] = *reinterpret_cast<bf16x8 *>(&v);
        }
    }
    // rows of a tree's mask are asked for here and looked at behind the first pages' loads (on the device, us, looked at here and so: five drafts of four chats of
    // 8/2/64 5.4, 5.2; seven of 48 sequences of 32/8/128 e4m3 27.7, 26.7)
    uint64_t bits[NT][PKV_TREE_WORDS];
    if constexpr (TREE) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int i = 0; i < PKV_TREE_WORDS; ++i)      // (a column that stands for no query has the first token's)
                bits[c][i] = mk.sees[(size_t)(u.first + tok[c]) * mk.words + (i < mk.words ? i : mk.words - 1)];
    }
    int ctx = PKV_CONST(int32_t, d.ctx_lens)[u.seq], cap = PKV_CONST(int32_t, d.row_len)[u.seq];
    asm volatile("" : "+s"(ctx), "+s"(cap));              // both at once
    cap *= PKV_T;
    // what this lane's columns see, in tokens of the row
    const int window = mk.window;
    int base = 0, hi[NT], lo[NT], L, lo_first, lo_last, hi_first;
    uint32_t *mask_row[NT];
    if constexpr (TREE) {
        base = ctx - u.chunk;
        L = base < 0 ? 0 : (ctx < cap ? ctx : cap);
        lo_first = base + 1 - window;
        lo_last = base + u.chunk - window;
        hi_first = base;
    } else {
        L = ctx < 0 ? 0 : (ctx < cap ? ctx : cap);
        const int pos0 = L - u.chunk + u.chunk0;          // of the unit's first query
        L = pos0 + u.tokens;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            hi[c] = pos0 + tok[c] + 1;
            lo[c] = hi[c] - window;
        }
        lo_first = pos0 + 1 - window;
        lo_last = L - window;
        hi_first = pos0 + 1;
    }
    const Walk walk = walk_of(L, lo_first, lo_last, hi_first, mk.sinks);
    const int shift = walk.skip * PKV_T;
    base -= shift;
    if constexpr (!TREE) {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            hi[c] -= shift;
            lo[c] -= shift;
        }
    }
    auto tree_masks = [&]() __attribute__((always_inline)) {
        if constexpr (TREE) {
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                int seen = 0;
                mask_row[c] = s_mask + (w * MC + tok[c]) * MASK_WORDS;
#pragma unroll
                for (int i = 0; i < PKV_TREE_WORDS; ++i)
                    if (i < mk.words) {
                        const int left = u.chunk - 64 * i;
                        seen += __popcll(bits[c][i] & (left >= 64 ? ~0ull : (left <= 0 ? 0ull : (1ull << left) - 1ull)));
                        mask_row[c][2 * i] = (uint32_t)bits[c][i];
                        mask_row[c][2 * i + 1] = (uint32_t)(bits[c][i] >> 32);
                    }
                hi[c] = base;
                lo[c] = base + (seen > 0 ? seen : 1) - window;
            }
        }
    };
    const int n_pages = walk.pages(), max_parts = u.parts;
    constexpr int STEP = 2 * SMALL_WAVES;
    // as many parts of equal length as the host asked for, but none shorter than u.size
    int size = (n_pages + max_parts - 1) / max_parts;
    size = (size + STEP - 1) / STEP * STEP;
    size = size < u.size ? u.size : size;
    const int n_parts = n_pages > size ? (n_pages + size - 1) / size : 1;
    if (u.part >= n_parts) return;
    const int page0 = u.part * size + 2 * w, pe = (u.part + 1) * size < n_pages ? (u.part + 1) * size : n_pages;
    State<D, DT> st[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) {
#pragma unroll
        for (int jt = 0; jt < TL::NV; ++jt) st[c].acc[jt] = f32x4{0.f, 0.f, 0.f, 0.f};
        st[c].m = -INFINITY;
        st[c].l = 0.f;
    }

    // This wave's pairs: pages page0 + STEP k and the one behind it.  Lane i works out where page i & 1 of pair window + (i >> 1) is.
    bool bad = false;
    uint32_t addr_lo = 0, addr_hi = 0, records = 0;
    float page_sk = 0.f, page_sv = 0.f;
    int pair0 = 0;                                        // the lanes' pages are those of pairs pair0 .. pair0 + 31
    auto locate = [&](int k) __attribute__((always_inline)) {
        pair0 = k;
        const int i = page0 + STEP * (k + (lane >> 1)) + (lane & 1), page = walk.page(i);
        const uint32_t id = (uint32_t)row[page < d.row_stride ? page : d.row_stride - 1];
        const bool in_pool = id < d.max_block_id, live = i < pe;
        bad |= live && !in_pool;
        const uint8_t *blk = block_ptr(d, id);
        if (DT == PKV_E4M3) {
            const float *hdr = reinterpret_cast<const float *>(live && in_pool ? blk : reinterpret_cast<const uint8_t *>(d.safe));
            page_sk = hdr[u.kvh];
            page_sv = hdr[d.Hkv + u.kvh];
            blk += PKV_FP8_HEADER;
        }
        blk += (size_t)u.kvh * 2 * TL::TILE_BYTES;
        addr_lo = (uint32_t)(uintptr_t)blk;
        addr_hi = (uint32_t)((uintptr_t)blk >> 32);
        records = live && in_pool ? 2 * TL::TILE_BYTES : 0;
    };
    auto lane_of = [&](uint32_t x, int at) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readlane((int)x, at); };
    auto tiles = [&](int k, int half) __attribute__((always_inline)) {
        const int at = 2 * (k - pair0) + half;
        return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<uint8_t *>(lane_of(addr_lo, at) | (uint64_t)lane_of(addr_hi, at) << 32), 0,
                                                 (int)lane_of(records, at), 0x00020000);
    };
    const int voff = lane * 16;
    auto load = [&](u32x4 *r, __amdgpu_buffer_rsrc_t rsrc, int at) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < TL::NL; ++j) r[j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff + j * 1024, at, 2 /* non-temporal */);
        asm volatile("" ::: "memory");                    // in this order everywhere: loads in flight are counted
    };
    auto scale_of = [&](float x, int k, int half) __attribute__((always_inline)) { return __uint_as_float(lane_of(__float_as_uint(x), 2 * (k - pair0) + half)); };
    // Scores of pair k's 32 tokens, scaled and masked, as the columns' softmax takes them; `r`'s V is blanked where no query sees it.
    // (Whether masks are needed is decided ahead of the products, and without branches: the compiler waits for a product's result along one of two
    // ways that part behind it and meet where it is read, and not along the other.)
    auto scores = [&](float (*s)[8], const PairRegs<D, DT> &r) __attribute__((always_inline)) {
        const float sca = DT == PKV_E4M3 ? d.scale_log2 * r.a.sk : d.scale_log2, scb = DT == PKV_E4M3 ? d.scale_log2 * r.b.sk : d.scale_log2;
        f32x4 sa[NT], sb[NT];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            sa[c] = qk_page<D, DT>(r.a, qf[c]);
            sb[c] = qk_page<D, DT>(r.b, qf[c]);
        }
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[c][i] = sa[c][i] * sca;
                s[c][4 + i] = sb[c][i] * scb;
            }
    };
    auto pair_is_masked = [&](int k) __attribute__((always_inline)) {
        const int p = page0 + STEP * k;
        return !walk.plain(PKV_T * p) | !(p + 1 < pe);
    };
    auto there = [&](int k) __attribute__((always_inline)) {          // tokens of pair k that are in the part
        const int p = page0 + STEP * k;
        return below(walk.len - PKV_T * p) & (p + 1 < pe ? 0xffffffffu : 0xffffu);
    };
    auto sees = [&](int c, int k) __attribute__((always_inline)) {    // of those, the ones that this lane's column of tile c sees
        const int x0 = PKV_T * (page0 + STEP * k);
        uint32_t mine = seen_bits(x0, hi[c], lo[c], walk.sinks);
        if constexpr (TREE) mine |= row_bits(mask_row[c], 2 * mk.words, x0 - base);
        return mine & there(k);
    };
    auto mask_scores = [&](float (*s)[8], int k) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            const uint32_t mine = sees(c, k) >> (4 * G);
#pragma unroll
            for (int i = 0; i < 4; ++i) {                  // (a select, so that a NaN logit of an unseen token cannot leak)
                if (!(mine >> i & 1u)) s[c][i] = -INFINITY;
                if (!(mine >> (16 + i) & 1u)) s[c][4 + i] = -INFINITY;
            }
        }
    };
    auto mask_v = [&](PairRegs<D, DT> &r, int k) __attribute__((always_inline)) {
        const uint32_t any = (there(k) & walk.some(PKV_T * (page0 + STEP * k))) >> (4 * G);
        keep_v<D, DT>(r.a.v, any);
        keep_v<D, DT>(r.b.v, any >> 16);
    };
    auto products = [&](const PairRegs<D, DT> &r, const bf16x8 *ph, const bf16x8 *pl) __attribute__((always_inline)) {
#pragma unroll
        for (int jt = 0; jt < TL::NV; ++jt) {
            const u32x2 va = v_half<D, DT>(r.a, jt), vb = v_half<D, DT>(r.b, jt);
            const bf16x8 av = as_bf16x8(mk4(va.x, va.y, vb.x, vb.y));
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                st[c].acc[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, ph[c], st[c].acc[jt], 0, 0, 0);
                st[c].acc[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, pl[c], st[c].acc[jt], 0, 0, 0);
            }
        }
    };
    const int n_pairs = page0 < pe ? (pe - page0 + STEP - 1) / STEP : 0;
    if constexpr (NT == 1) {
        auto load_pair = [&](PairRegs<D, DT> &r, int k) __attribute__((always_inline)) {
            const __amdgpu_buffer_rsrc_t a = tiles(k, 0), b = tiles(k, 1);
            load(r.a.k, a, 0);
            load(r.a.v, a, TL::TILE_BYTES);
            load(r.b.k, b, 0);
            load(r.b.v, b, TL::TILE_BYTES);
            if (DT == PKV_E4M3) {
                r.a.sk = scale_of(page_sk, k, 0);
                r.a.sv = scale_of(page_sv, k, 0);
                r.b.sk = scale_of(page_sk, k, 1);
                r.b.sv = scale_of(page_sv, k, 1);
            }
        };
        auto step = [&](PairRegs<D, DT> &r, PairRegs<D, DT> &o, int k, bool more) __attribute__((always_inline)) {
            if (more) load_pair(o, k + 1);
            const bool masked = pair_is_masked(k);
            float s[NT][8];
            scores(s, r);
            if (masked) {                                 // a branch of its own
                mask_scores(s, k);
                mask_v(r, k);
            }
            bf16x8 ph[NT], pl[NT];
            softmax_pair<D, DT>(st[0], s[0], r.a.sv, r.b.sv, ph[0], pl[0]);
            products(r, ph, pl);
        };
        if (n_pairs > 0) {
            PairRegs<D, DT> ring[2];
            locate(0);
            load_pair(ring[0], 0);
            tree_masks();
            int k = 0;
            if (n_pairs > 1) {
                do {
                    if (k + 2 - pair0 >= 32) locate(k + 1);
                    step(ring[0], ring[1], k, true);
                    step(ring[1], ring[0], k + 1, true);
                    k += 2;
                } while (k + 2 <= n_pairs);
            }
            if (k < n_pairs) step(ring[0], ring[1], k, false);
        }
    } else if (n_pairs > 0) {
        PairRegs<D, DT> r;
        auto load_k = [&](int k) __attribute__((always_inline)) {
            load(r.a.k, tiles(k, 0), 0);
            load(r.b.k, tiles(k, 1), 0);
            r.a.sk = DT == PKV_E4M3 ? scale_of(page_sk, k, 0) : 0.f;
            r.b.sk = DT == PKV_E4M3 ? scale_of(page_sk, k, 1) : 0.f;
        };
        auto load_v = [&](int k) __attribute__((always_inline)) {
            load(r.a.v, tiles(k, 0), TL::TILE_BYTES);
            load(r.b.v, tiles(k, 1), TL::TILE_BYTES);
            r.a.sv = DT == PKV_E4M3 ? scale_of(page_sv, k, 0) : 0.f;
            r.b.sv = DT == PKV_E4M3 ? scale_of(page_sv, k, 1) : 0.f;
        };
        locate(0);
        load_k(0);
        load_v(0);
        tree_masks();
        for (int k = 0; k < n_pairs; ++k) {
            if (k + 1 - pair0 >= 32) locate(k + 1);
            const bool masked = pair_is_masked(k);
            float s[NT][8];
            scores(s, r);
            load_k(k + 1);                                // (a pair behind the part's last has no records: nothing is read)
            if (masked) mask_scores(s, k);
            bf16x8 ph[NT], pl[NT];
#pragma unroll
            for (int c = 0; c < NT; ++c) softmax_pair<D, DT>(st[c], s[c], r.a.sv, r.b.sv, ph[c], pl[c]);
            if (masked) mask_v(r, k);
            products(r, ph, pl);
            load_v(k + 1);
        }
    }
    // once more, if sums are not finite (mask_walk.h)
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int jt = 0; jt < TL::NV; ++jt) sum += (st[c].acc[jt][0] + st[c].acc[jt][1]) + (st[c].acc[jt][2] + st[c].acc[jt][3]);
    if (__builtin_expect(__any(!is_finite(sum)), 0)) {
#pragma unroll
        for (int c = 0; c < NT; ++c) {
#pragma unroll
            for (int jt = 0; jt < TL::NV; ++jt) st[c].acc[jt] = f32x4{0.f, 0.f, 0.f, 0.f};
            st[c].m = -INFINITY;
            st[c].l = 0.f;
        }
#pragma unroll 1
        for (int k = 0; k < n_pairs; ++k) {
            if (k % 32 == 0) locate(k);
            PairRegs<D, DT> r;
            load(r.a.k, tiles(k, 0), 0);
            load(r.b.k, tiles(k, 1), 0);
            load(r.a.v, tiles(k, 0), TL::TILE_BYTES);
            load(r.b.v, tiles(k, 1), TL::TILE_BYTES);
            if (DT == PKV_E4M3) {
                r.a.sk = scale_of(page_sk, k, 0);
                r.a.sv = scale_of(page_sv, k, 0);
                r.b.sk = scale_of(page_sk, k, 1);
                r.b.sv = scale_of(page_sv, k, 1);
            }
            float s[NT][8];
            scores(s, r);
            mask_scores(s, k);
            bf16x8 ph[NT], pl[NT];
            u32x4 mine[NT];
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const uint32_t bits = sees(c, k) >> (4 * G);
                mine[c] = mk4(halves_of(bits), halves_of(bits >> 2), halves_of(bits >> 16), halves_of(bits >> 18));
                softmax_pair<D, DT>(st[c], s[c], r.a.sv, r.b.sv, ph[c], pl[c]);
                ph[c] = as_bf16x8(__builtin_bit_cast(u32x4, ph[c]) & mine[c]);       // (a block's scale may be none, too)
                pl[c] = as_bf16x8(__builtin_bit_cast(u32x4, pl[c]) & mine[c]);
            }
            mask_v(r, k);
#pragma unroll
            for (int jt = 0; jt < TL::NV; ++jt) {
                const u32x2 va = v_half<D, DT>(r.a, jt), vb = v_half<D, DT>(r.b, jt);
                const u32x4 off = mk4(strange_halves(va.x), strange_halves(va.y), strange_halves(vb.x), strange_halves(vb.y)) & kSpoil;
#pragma unroll
                for (int c = 0; c < NT; ++c) {
                    st[c].acc[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(off), as_bf16x8(mine[c] & kSpoil), st[c].acc[jt], 0, 0, 0);
                    st[c].acc[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(off), as_bf16x8(mine[c] & kMinusSpoil), st[c].acc[jt], 0, 0, 0);
                }
            }
#pragma unroll
            for (int j = 0; j < TL::NL; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    r.a.v[j][i] = finite_only<DT>(r.a.v[j][i]);
                    r.b.v[j][i] = finite_only<DT>(r.b.v[j][i]);
                }
            products(r, ph, pl);
        }
    }
#pragma unroll
    for (int c = 0; c < NT; ++c) {
        float l = st[c].l;
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const int col = 16 * c + n;
        if (col < cols) {
            float *a = s_acc + (w * cols + col) * D;
#pragma unroll
            for (int jt = 0; jt < TL::NV; ++jt) *reinterpret_cast<f32x4 *>(a + 16 * jt + 4 * G) = st[c].acc[jt];
            if (G == 0) {
                s_m[w * MC + col] = st[c].m;
                s_l[w * MC + col] = l;
            }
        }
    }
    if (__any(bad) && lane == 0) atomicOr(d.err, 1u);
    __syncthreads();
    // the sums of the work-group: lane by lane four output elements of one column
    const int quads = cols * (D / 4);
    const bool whole = n_parts == 1;
    float *mine = d.ws + u.partial + u.part * u.step;
    float *out = d.out + ((size_t)u.first * d.Hq + u.kvh * g) * D;
    for (int i = threadIdx.x; i < quads; i += 64 * SMALL_WAVES) {
        const int c = i / (D / 4), x = i - c * (D / 4), t = c / g;
        float M = s_m[c];
#pragma unroll
        for (int v = 1; v < SMALL_WAVES; ++v) M = fmaxf(M, s_m[v * MC + c]);
        float den = 0.f;
        f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < SMALL_WAVES; ++v) {
            const float f = merge_weight(s_m[v * MC + c], M);
            den += f * s_l[v * MC + c];
            num += f * *reinterpret_cast<const f32x4 *>(s_acc + (v * cols + c) * D + 4 * x);
        }
        if (whole) {
            *reinterpret_cast<f32x4 *>(out + ((size_t)t * d.Hq + c - t * g) * D + 4 * x) = den != 0.f ? num * (1.0f / den) : num;
        } else {
            *reinterpret_cast<f32x4 *>(mine + c * D + 4 * x) = num;
            if (x == 0) {
                mine[cols * D + c] = M;
                mine[cols * D + cols + c] = den;
            }
        }
    }
    if (whole) return;
    // partials and counters are in uncached memory: the order of a wave's own accesses is all there is to enforce
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) *s_arrived = atomicAdd(d.cnt + u.slot, 1u);
    __syncthreads();
    if (*s_arrived != (uint32_t)(n_parts - 1)) return;
    if (threadIdx.x == 0) d.cnt[u.slot] = 0u;             // ready for the next launch
    const float *first = d.ws + u.partial;
    auto part_sums = [&](f32x4 *v, int c0, int c, int x) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = *reinterpret_cast<const f32x4 *>(first + (size_t)(c0 + k < n_parts ? c0 + k : n_parts - 1) * u.step + c * D + 4 * x);
    };
    f32x4 v[8];
    {
        const int i = (int)threadIdx.x < quads ? (int)threadIdx.x : quads - 1, c = i / (D / 4);
        part_sums(v, 0, c, i - c * (D / 4));
    }
    for (int i = threadIdx.x; i < n_parts * cols; i += 64 * SMALL_WAVES) {
        const int p = i / cols, c = i - p * cols;
        s_acc[i] = first[(size_t)p * u.step + cols * D + c];
        s_acc[MAX_PIECES * MC + i] = first[(size_t)p * u.step + cols * D + cols + c];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < quads; i += 64 * SMALL_WAVES) {
        const int c = i / (D / 4), x = i - c * (D / 4), t = c / g;
        float M = -INFINITY, den = 0.f;
        f32x4 num = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < n_parts; ++p) M = fmaxf(M, s_acc[p * cols + c]);
        for (int p0 = 0; p0 < n_parts; p0 += 8) {
            if (p0 > 0 || i >= 64 * SMALL_WAVES) part_sums(v, p0, c, x);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (p0 + k < n_parts) {
                    const float f = merge_weight(s_acc[(p0 + k) * cols + c], M);
                    den += f * s_acc[MAX_PIECES * MC + (p0 + k) * cols + c];
                    num += f * v[k];
                }
        }
        *reinterpret_cast<f32x4 *>(out + ((size_t)t * d.Hq + c - t * g) * D + 4 * x) = den != 0.f ? num * (1.0f / den) : num;
    }
}

}  // namespace
