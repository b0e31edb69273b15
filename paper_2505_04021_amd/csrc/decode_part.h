// Decode attention's page pairs, softmax steps and the work-group that walks one part of a (sequence, kv head) (gfx950).
// attn_kernels.hip says what the layout and the mapping are.
#pragma once
#include "mfma_util.h"

namespace {

constexpr int T = PKV_T;

template <int D, int DT>
struct Tile {
    static constexpr int E = DT == PKV_BF16 ? 2 : 1;
    static constexpr int TILE_BYTES = T * D * E;           // one K or V tile
    static constexpr int NL = TILE_BYTES / 1024;           // 16-byte loads per lane per tile
    static constexpr int NK = D / 32;                      // QK^T MFMAs per page
    static constexpr int NV = D / 16;                      // d-tiles of the output
};

template <int D, int DT>
struct PageRegs {
    u32x4 k[Tile<D, DT>::NL];
    u32x4 v[Tile<D, DT>::NL];
    float sk, sv;
};

// Block ids of a page pair.  They are read through the scalar cache one step before the
// loads that need them are issued, so the latency of this dependent access (block table
// -> address -> K/V load) is covered by the arithmetic of the step in between.
struct PairIds {
    uint32_t a, b;
};

__device__ __forceinline__ PairIds fetch_ids(const AttnDesc &d, const int32_t *row, int page) {
    const int last = d.row_stride - 1;
    // wave-uniform, and said to be: the ids come through the scalar cache (a vector load would wait for all K and V in flight)
    row = reinterpret_cast<const int32_t *>((uint32_t)__builtin_amdgcn_readfirstlane((int)(uintptr_t)row) |
                                            (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uintptr_t)row >> 32)) << 32);
    const int ia = page < last ? page : last, ib = page + 1 < last ? page + 1 : last;
    PairIds ids;
    ids.a = (uint32_t)__builtin_amdgcn_readfirstlane(PKV_CONST(int32_t, row)[ia]);
    ids.b = (uint32_t)__builtin_amdgcn_readfirstlane(PKV_CONST(int32_t, row)[ib]);
    return ids;
}

// Issue the loads of one page (K tile, V tile) of one kv head.  Buffer loads with a
// per-page resource descriptor: a page beyond the chunk (live == false) gets a
// descriptor of zero records, so its loads return zeros without touching memory.
// That keeps every load of the software pipeline unconditional, which lets the
// compiler count outstanding loads exactly (s_waitcnt vmcnt(N) with N > 0) instead of
// draining the queue at each control-flow join.
template <int D, int DT>
__device__ __forceinline__ void load_page(PageRegs<D, DT> &r, const AttnDesc &d, uint32_t id, bool live, int kvh,
                                          int lane, uint32_t &bad) {
    using TL = Tile<D, DT>;
    if (id >= d.max_block_id) {          // never dereference an id outside the pool
        bad |= live ? 1u : 0u;           // reported once, after the last load (no store inside the loop)
        id = 0;
        live = false;                    // the page is skipped: frame 0 need not even be backed by memory
    }
    const uint8_t *blk = block_ptr(d, id);
    if (DT == PKV_E4M3) {
        // A dead page's id is whatever the table holds past the row's end: possibly a block of a
        // frame that was given back and, in an elastic pool, is no longer backed by memory.
        // Its header must not be read (the tile loads below are harmless: zero records).
        const float *hdr = reinterpret_cast<const float *>(live ? blk : reinterpret_cast<const uint8_t *>(d.safe));
        r.sk = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(PKV_CONST(float, hdr)[kvh])));
        r.sv = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(PKV_CONST(float, hdr)[d.Hkv + kvh])));
        if (!live) r.sk = r.sv = 0.f;
        blk += PKV_FP8_HEADER;
    }
    const uint8_t *tiles = blk + (size_t)kvh * 2 * TL::TILE_BYTES;
    const __amdgpu_buffer_rsrc_t rsrc =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(tiles), 0, live ? 2 * TL::TILE_BYTES : 0, 0x00020000);
    const int voff = lane * 16;
#pragma unroll
    for (int j = 0; j < TL::NL; ++j)
        r.k[j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff + j * 1024, 0, 2 /* non-temporal */);
#pragma unroll
    for (int j = 0; j < TL::NL; ++j)
        r.v[j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff + j * 1024, TL::TILE_BYTES, 2);
}

template <int D, int DT>
struct State {
    f32x4 acc[Tile<D, DT>::NV];   // out^T tiles: acc[jt][i] = out[16jt + 4G + i][head n]
    float m, l;                   // running max (log2 domain) and this lane's share of the sum
};

// Two consecutive pages of a piece travel and are processed together (32 tokens): one
// max / rescale step per 32 tokens and 16x16x32 MFMAs for the PV product.
template <int D, int DT>
struct PairRegs {
    PageRegs<D, DT> a, b;
};

template <int D, int DT>
__device__ __forceinline__ void load_pair(PairRegs<D, DT> &r, const AttnDesc &d, PairIds ids, bool live_a, bool live_b,
                                          int kvh, int lane, uint32_t &bad) {
    load_page<D, DT>(r.a, d, ids.a, live_a, kvh, lane, bad);
    load_page<D, DT>(r.b, d, ids.b, live_b, kvh, lane, bad);
}

// S[token][head] of one page: K (A operand, row = token) times q (B operand)
template <int D, int DT>
__device__ __forceinline__ f32x4 qk_page(const PageRegs<D, DT> &r, const bf16x8 *qf) {
    using TL = Tile<D, DT>;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (DT == PKV_BF16) {
#pragma unroll
        for (int j = 0; j < TL::NK; ++j) {
            u32x4 kv = r.k[j];
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<bf16x8 *>(&kv), qf[j], s, 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int j2 = 0; j2 < TL::NL; ++j2) {
            const u32x4 kv = r.k[j2];
            const u32x2 a0 = fp8x4_to_bf16x4(kv.x), a1 = fp8x4_to_bf16x4(kv.y);
            const u32x2 b0 = fp8x4_to_bf16x4(kv.z), b1 = fp8x4_to_bf16x4(kv.w);
            u32x4 ka = mk4(a0.x, a0.y, a1.x, a1.y);
            u32x4 kb = mk4(b0.x, b0.y, b1.x, b1.y);
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<bf16x8 *>(&ka), qf[2 * j2], s, 0, 0, 0);
            s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<bf16x8 *>(&kb), qf[2 * j2 + 1], s, 0, 0, 0);
        }
    }
    return s;
}

// V of one page for output tile jt as four bf16: V[4G..4G+3][16jt + (lane & 15)]
template <int D, int DT>
__device__ __forceinline__ u32x2 v_half(const PageRegs<D, DT> &r, int jt) {
    if (DT == PKV_BF16) {
        const u32x4 vv = r.v[jt >> 1];
        return (jt & 1) ? mk2(vv.z, vv.w) : mk2(vv.x, vv.y);
    }
    const u32x4 vv = r.v[jt >> 2];
    const uint32_t w = (jt & 3) == 0 ? vv.x : (jt & 3) == 1 ? vv.y : (jt & 3) == 2 ? vv.z : vv.w;
    return fp8x4_to_bf16x4(w);
}

// bf16 hi + lo of four probabilities: 16 significant bits reach the matrix unit
__device__ __forceinline__ void split_p(const float *p, u32x2 &hi, u32x2 &lo) {
    const uint32_t h01 = pack_bf16_rne(p[0], p[1]), h23 = pack_bf16_rne(p[2], p[3]);
    const float l0 = p[0] - __uint_as_float(h01 << 16), l1 = p[1] - __uint_as_float(h01 & 0xffff0000u);
    const float l2 = p[2] - __uint_as_float(h23 << 16), l3 = p[3] - __uint_as_float(h23 & 0xffff0000u);
    hi = mk2(h01, h23);
    lo = mk2(pack_bf16_rne(l0, l1), pack_bf16_rne(l2, l3));
}

// Blanks the tokens of a V tile past the context, which may hold anything (even NaN); live of the four that this lane holds count.
template <int D, int DT>
__device__ __forceinline__ void blank_v(u32x4 *v, int live) {
    const uint32_t m01 = live >= 2 ? 0xffffffffu : (live == 1 ? 0x0000ffffu : 0u), m23 = live >= 4 ? 0xffffffffu : (live == 3 ? 0x0000ffffu : 0u);
    const uint32_t m = live >= 4 ? 0xffffffffu : (live <= 0 ? 0u : (1u << (8 * live)) - 1u);      // codes
#pragma unroll
    for (int j = 0; j < Tile<D, DT>::NL; ++j) v[j] &= DT == PKV_BF16 ? mk4(m01, m23, m01, m23) : mk4(m, m, m, m);
}

// Small launches: the reference point, the sums and the probabilities of one online-softmax step, as process_pair below takes them,
// from scaled and masked logits s; but logits of -inf may be all that a column has seen so far, and weigh nothing.
template <int D, int DT>
__device__ __forceinline__ void softmax_pair(State<D, DT> &st, const float *s, float sva, float svb, bf16x8 &phv, bf16x8 &plv) {
    using TL = Tile<D, DT>;
    float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    mx = rows_max(mx);
    const float m_new = fmaxf(st.m, mx);
    // wave-uniform: the reference point of the exponentials moves, and the sums are rescaled, only when some
    // column's maximum has run ahead of it by more than kRescaleSlack (probabilities stay below 2^kRescaleSlack)
    if (__any(m_new > st.m + kRescaleSlack)) {
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - m_new);
        st.l *= alpha;
#pragma unroll
        for (int jt = 0; jt < TL::NV; ++jt) st.acc[jt] *= alpha;
        st.m = m_new;
    }
    float p[8];
    const float m_ref = st.m == -INFINITY ? 0.f : st.m;      // then every s is -inf and every p is 0
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(s[i] - m_ref);
    st.l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    if (DT == PKV_E4M3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] *= sva;
            p[4 + i] *= svb;
        }
    }
    // B operand of the PV product: lane (G, head) holds P for tokens 4G..4G+3 of page a, then of page b
    u32x2 ha, la, hb, lb;
    split_p(p, ha, la);
    split_p(p + 4, hb, lb);
    u32x4 ph = mk4(ha.x, ha.y, hb.x, hb.y), pl = mk4(la.x, la.y, lb.x, lb.y);
    phv = *reinterpret_cast<bf16x8 *>(&ph);
    plv = *reinterpret_cast<bf16x8 *>(&pl);
}

// One online-softmax step over the 32 tokens of a page pair.  valid_a is 1..16,
// valid_b 0..16 (0: the pair has no second page; its registers hold zeros).  Whether the
// pair needs masks is decided at run time inside (one code path with selects: the kernel is
// bound by memory).
template <int D, int DT>
__device__ __forceinline__ void process_pair(State<D, DT> &st, const PairRegs<D, DT> &r, const bf16x8 *qf,
                                             float scale_log2, int valid_a, int valid_b, int G) {
    using TL = Tile<D, DT>;
    const bool tail = valid_a < T || valid_b < T;
    f32x4 sa = qk_page<D, DT>(r.a, qf);
    f32x4 sb = qk_page<D, DT>(r.b, qf);
    const float sca = DT == PKV_E4M3 ? scale_log2 * r.a.sk : scale_log2;
    const float scb = DT == PKV_E4M3 ? scale_log2 * r.b.sk : scale_log2;
    float s[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = sa[i] * sca;
        s[4 + i] = sb[i] * scb;
        if (tail) {                                        // select, so a NaN logit of a dead token cannot leak
            if (4 * G + i >= valid_a) s[i] = -INFINITY;
            if (4 * G + i >= valid_b) s[4 + i] = -INFINITY;
        }
    }
    float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    mx = rows_max(mx);
    const float m_new = fmaxf(st.m, mx);
    // wave-uniform: the reference point of the exponentials moves, and the sums are rescaled, only when some
    // column's maximum has run ahead of it by more than kRescaleSlack (probabilities stay below 2^kRescaleSlack)
    if (__any(m_new > st.m + kRescaleSlack)) {
        const float alpha = __builtin_amdgcn_exp2f(st.m - m_new);
        st.l *= alpha;
#pragma unroll
        for (int jt = 0; jt < TL::NV; ++jt) st.acc[jt] *= alpha;
        st.m = m_new;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(s[i] - st.m);
    st.l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    if (DT == PKV_E4M3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] *= r.a.sv;
            p[4 + i] *= r.b.sv;
        }
    }
    // B operand of the PV product: lane (G, head) holds P for tokens 4G..4G+3 of page a, then of page b
    u32x2 ha, la, hb, lb;
    split_p(p, ha, la);
    split_p(p + 4, hb, lb);
    u32x4 ph = mk4(ha.x, ha.y, hb.x, hb.y), pl = mk4(la.x, la.y, lb.x, lb.y);
    const bf16x8 phv = *reinterpret_cast<bf16x8 *>(&ph), plv = *reinterpret_cast<bf16x8 *>(&pl);
    // tokens past the context length may hold anything (even NaN): blank their V
    uint32_t ma01 = 0xffffffffu, ma23 = 0xffffffffu, mb01 = 0xffffffffu, mb23 = 0xffffffffu;
    if (tail) {
        const int la_ = valid_a - 4 * G, lb_ = valid_b - 4 * G;
        ma01 = la_ >= 2 ? 0xffffffffu : (la_ == 1 ? 0x0000ffffu : 0u);
        ma23 = la_ >= 4 ? 0xffffffffu : (la_ == 3 ? 0x0000ffffu : 0u);
        mb01 = lb_ >= 2 ? 0xffffffffu : (lb_ == 1 ? 0x0000ffffu : 0u);
        mb23 = lb_ >= 4 ? 0xffffffffu : (lb_ == 3 ? 0x0000ffffu : 0u);
    }
#pragma unroll
    for (int jt = 0; jt < TL::NV; ++jt) {
        // A operand: V^T, row = output element 16jt + (lane & 15), k = the same eight tokens
        const u32x2 va = v_half<D, DT>(r.a, jt), vb = v_half<D, DT>(r.b, jt);
        u32x4 vv = tail ? mk4(va.x & ma01, va.y & ma23, vb.x & mb01, vb.y & mb23) : mk4(va.x, va.y, vb.x, vb.y);
        const bf16x8 av = *reinterpret_cast<bf16x8 *>(&vv);
        st.acc[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, phv, st.acc[jt], 0, 0, 0);
        st.acc[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, plv, st.acc[jt], 0, 0, 0);
    }
}

constexpr int FLIGHT_KIB_2WAVES = 16;      // bytes in flight per wave, two waves per SIMD
// Page pairs resident per wave: one in use, the rest in flight.  In the form with two waves per
// SIMD every shape keeps the same number of bytes in flight (FLIGHT_KIB_2WAVES), small pages
// through a deeper ring; otherwise waves of a small-page model would fall behind the others in
// a grouped launch.
template <int D, int DT, int FLIGHT_KIB = FLIGHT_KIB_2WAVES>
struct Ring {
    static constexpr int PAIR_BYTES = 4 * Tile<D, DT>::TILE_BYTES;        // K and V tiles of two pages
    static constexpr int N = 1 + (FLIGHT_KIB * 1024 + PAIR_BYTES - 1) / PAIR_BYTES;
};
// The second form of the kernel: one wave per SIMD, the host launching only as many waves as it
// takes to keep the memory system busy (512 for bf16 pages of 8 KiB).  A wave alone on its SIMD
// turns a page pair over in 0.7-1.1 us whatever it has in flight, so one pair in use and one
// travelling is all the ring needs (8 KiB covers a pair of every shape but bf16 with 128-wide
// heads, whose pair of 16 KiB is the one in flight anyway); more bytes outstanding only lengthen
// the queues in front of the memory channels, and the launch as a whole gets slower.
constexpr int FLIGHT_KIB_1WAVE = 8;
constexpr int MAX_PIECES = 64;   // pieces of one (sequence, kv head) the merge stages in LDS

__device__ __forceinline__ int ctx_clamped(const AttnDesc &d, int seq) {
    int L = PKV_CONST(int32_t, d.ctx_lens)[seq];
    const int cap = (d.row_len ? PKV_CONST(int32_t, d.row_len)[seq] : d.row_stride) * T;
    return L < 0 ? 0 : (L > cap ? cap : L);
}

// Whether MFMA column n is a query head at all.  Worked out anew for every piece: known to be the same throughout,
// the compiler splits the streaming loop on it and loses count of the loads in flight (full waits inside the loop).
__device__ __forceinline__ bool column_live(const AttnDesc &d, int n) {
    asm volatile("" : "+v"(n));
    return n < d.g;
}

// q as the B operand (column n: head n of the kv head's group): lane (G, n) holds q[column n][8(4j+G) .. +7] for each k-step j
template <int D>
__device__ __forceinline__ void load_q(bf16x8 *qf, const AttnDesc &d, int seq, int kvh, int lane) {
    const int G = lane >> 4, n = lane & 15;
    const uint16_t *qrow = d.q + ((size_t)seq * d.Hq + kvh * d.g + n) * D;
    const bool live = column_live(d, n);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        u32x4 v = mk4(0, 0, 0, 0);
        if (live) v = *reinterpret_cast<const u32x4 *>(qrow + 8 * (4 * j + G));
        qf[j] = *reinterpret_cast<bf16x8 *>(&v);
    }
}

// Small launches: one work-group of SMALL_WAVES waves per part of a (sequence, kv head).
//
// Such a launch is bound by the number of dependent memory trips, not by bytes: the kernels above find their share from
// all context lengths, then its block ids, then the pages, and hand every cut segment over through memory (partial,
// arrival, partials of the others: three more trips of about 1 us).  Here the block index alone names the segment and
// the part, so block ids, context length and queries are asked for together and the pages behind them; the waves of
// the work-group take the part's page pairs in turn and join their sums through LDS.  Only segments longer than
// `part_pages` pages come in several parts, whose partials the last to arrive joins.  The host sizes the parts
// (plan_small); a context that has outgrown them (a launch replayed from a graph) gets longer parts here.
//
// A wave alone on its SIMD issues an instruction every four or five cycles, so once its pages are there it is bound by how many a
// page pair costs: with the addresses of both pages worked out by scalar instructions and masks in every pair some 410 (bf16) and
// 510 (e4m3, 128-wide heads), so 308 and 328 (cold branches included).  Us a launch, caches cold, with parts as they were and are
// chosen: 1 x 9735 tokens of 4/1/128 bf16 12.4, 11.8; 3 x 1717 of 2/1/128 e4m3 9.2, 8.1; 7 x 573 of 16/8/64 e4m3 7.3, 6.1; rows in one part
// 0.85 to 0.95 of the time before.  Eight waves a work-group instead of four take longer everywhere (2 x 767 of 16/4/128 9.2, 9.9).
constexpr int SMALL_WAVES = 4;

// Weight of a wave's sums with maximum m beside a joint maximum of M.  A wave that has seen nothing but logits of -inf has
// m = -inf and sums of zero (four waves each begin somewhere in the row, so that is not only the row's own start); so may
// have all waves of a part.
__device__ __forceinline__ float merge_weight(float m, float M) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M); }

// A part of a row for a kernel that joins the parts itself: which, of how many, of `size` pages, and where its sums go (per column D + 4
// floats: D sums, the reference point, the denominator).  Either the row of sequence `seq` with its queries, or its first `blocks` blocks with the
// queries of all `members`; columns: their heads, at most 16.
struct RowPart {
    int seq, kvh, part, parts, size, columns;
    int blocks, first;                // -1: the sequence's own row; its first one among the launch's members
    float *sums;
};

// The queries of a part's columns as load_q has them.
template <int D>
__device__ __forceinline__ void load_columns(bf16x8 *qf, const AttnDesc &d, const RowPart &at, const uint16_t *members, int lane) {
    const int G = lane >> 4, n = lane & 15, i = n / d.g;
    const bool live = n < at.columns;
    const int listed = (int)members[at.first + (live ? i : 0)], seq = at.blocks < 0 ? at.seq : listed;
    const uint16_t *qrow = d.q + ((size_t)seq * d.Hq + at.kvh * d.g + n - i * d.g) * D;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        u32x4 v = mk4(0, 0, 0, 0);
        if (live) v = *reinterpret_cast<const u32x4 *>(qrow + 8 * (4 * j + G));
        qf[j] = *reinterpret_cast<bf16x8 *>(&v);
    }
}

// PREFIXED: a row begins with the blocks of another one, shared[seq]; nothing but logits of -inf gives zeros.
template <int D, int DT, bool JOIN = true, bool PREFIXED = false>
__device__ __forceinline__ void attn_part(const AttnDesc &d, int wg, float *s_acc, float *s_m, float *s_l, uint32_t *s_arrived, const RowPart *at_part = nullptr,
                                          const uint16_t *members = nullptr, const SharedRow *shared = nullptr) {
    using TL = Tile<D, DT>;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int G = lane >> 4, n = lane & 15, g = JOIN ? d.g : at_part->columns;
    // Work-groups are dealt to the eight XCDs in turn.  With a multiple of eight kv heads these come fastest (each XCD
    // keeps its heads), then the parts of the row, then rows: eight lognormal rows of 2048 tokens take 22 us a launch, 27
    // with the parts slowest.  Otherwise parts come slowest, so that the first parts, which every row has, fall on all
    // XCDs (100 rows of 2 kv heads, parts before rows: 40 us, twice the ordinary form).
    int seq, kvh, part;
    if constexpr (!JOIN) {
        seq = at_part->seq;
        kvh = at_part->kvh;
        part = at_part->part;
    } else if ((d.Hkv & 7) == 0) {
        const int per_row = d.Hkv * d.parts, rest = wg % per_row;
        seq = wg / per_row;
        part = rest / d.Hkv;
        kvh = rest - part * d.Hkv;
    } else {
        const int n_segs = d.batch * d.Hkv, at = wg % n_segs;
        part = wg / n_segs;
        seq = at / d.Hkv;
        kvh = at - seq * d.Hkv;
    }
    const int seg = seq * d.Hkv + kvh;
    const int32_t *row = d.table + (size_t)seq * d.row_stride;
    bf16x8 qf[TL::NK];
    if constexpr (JOIN) load_q<D>(qf, d, seq, kvh, lane);
    else load_columns<D>(qf, d, *at_part, members, lane);
    // This wave's pairs: pages page0 + STEP k and the one behind it, k = 0, 1, ...  The ids of the first come by themselves, those of
    // the next 32 in one read, for any row; lane i works out where page i & 1 of pair 1 + (i >> 1) is, if there is a second pair.
    // All are asked for with the context length and the queries.
    constexpr int STEP = 2 * SMALL_WAVES;
    const int ahead = STEP * (lane >> 1) + (lane & 1);
    const int32_t *front = row;                           // PREFIXED: the row of its first blocks
    int n_front = 0;
    if constexpr (PREFIXED) {
        n_front = __builtin_amdgcn_readfirstlane(shared[seq].blocks);
        front = d.table + (size_t)__builtin_amdgcn_readfirstlane(shared[seq].row) * d.row_stride;
    }
    auto id_of = [&](int page) __attribute__((always_inline)) {
        if constexpr (PREFIXED) {
            const int at = page < n_front ? page : page - n_front;
            return (uint32_t)(page < n_front ? front : row)[at < d.row_stride ? at : d.row_stride - 1];
        }
        return (uint32_t)row[page < d.row_stride ? page : d.row_stride - 1];
    };
    auto pair_ids = [&](int page) __attribute__((always_inline)) {
        if constexpr (PREFIXED) {
            PairIds ids;
            ids.a = (uint32_t)__builtin_amdgcn_readfirstlane((int)id_of(page));
            ids.b = (uint32_t)__builtin_amdgcn_readfirstlane((int)id_of(page + 1));
            return ids;
        }
        return fetch_ids(d, row, page);
    };
    int page0 = part * (JOIN ? d.part_pages : at_part->size) + 2 * w;
    PairIds ids = pair_ids(page0);
    uint32_t id = id_of(page0 + STEP + ahead);
    int L;
    if constexpr (JOIN) L = __builtin_amdgcn_readfirstlane(ctx_clamped(d, seq));
    else if (at_part->blocks < 0) L = __builtin_amdgcn_readfirstlane(ctx_clamped(d, seq));
    else {
        // (no branch around the length: it would not be the same for all lanes any more in the compiler's eyes)
        const bool missing = PKV_CONST(int32_t, d.row_len)[seq] < at_part->blocks;       // the prefix is not there
        if (missing && threadIdx.x == 0) atomicOr(d.err, 1u);
        L = missing ? 0 : at_part->blocks * T;
    }
    if constexpr (PREFIXED) {
        const bool missing = n_front > 0 && PKV_CONST(int32_t, d.row_len)[shared[seq].row] < n_front;       // the prefix is not there: zero rows
        if (missing && threadIdx.x == 0) atomicOr(d.err, 1u);
        L = __builtin_amdgcn_readfirstlane(missing ? 0 : L + n_front * T);
    }
    const int n_pages = (L + T - 1) / T;
    int size = JOIN ? d.part_pages : at_part->size;
    if (n_pages > (JOIN ? d.parts : at_part->parts) * size) {                       // longer than the host knew
        size = (n_pages + (JOIN ? d.parts : at_part->parts) - 1) / (JOIN ? d.parts : at_part->parts);
        size = (size + STEP - 1) / STEP * STEP;
        page0 = part * size + 2 * w;
        ids = pair_ids(page0);
        id = id_of(page0 + STEP + ahead);
    }
    const int n_parts = n_pages > size ? (n_pages + size - 1) / size : 1;
    if (part >= n_parts) {
        if constexpr (!JOIN) {                            // (the join takes every part as it is, without a weight for those not written)
            for (int i = threadIdx.x; i < g * (D / 4 + 1); i += 64 * SMALL_WAVES)
                *reinterpret_cast<f32x4 *>(at_part->sums + 4 * i) = f32x4{i % (D / 4 + 1) == D / 4 ? -INFINITY : 0.f, 0.f, 0.f, 0.f};
        }
        return;
    }
    const int pe = (part + 1) * size < n_pages ? (part + 1) * size : n_pages;
    const int last_valid = L - (n_pages - 1) * T;
    State<D, DT> st;
#pragma unroll
    for (int jt = 0; jt < TL::NV; ++jt) st.acc[jt] = f32x4{0.f, 0.f, 0.f, 0.f};
    st.m = -INFINITY;
    st.l = 0.f;

    // where the tiles of this lane's page are, in how many bytes (none: the page is beyond the part, or its id outside the
    // pool, and is never read), and its scales
    bool bad = false;
    uint32_t addr_lo = 0, addr_hi = 0, records = 0;
    float page_sk = 0.f, page_sv = 0.f;
    auto locate = [&](int page, uint32_t id) __attribute__((always_inline)) {
        const bool in_pool = id < d.max_block_id, live = page < pe;
        bad |= live && !in_pool;
        const uint8_t *blk = block_ptr(d, id);
        if (DT == PKV_E4M3) {
            const float *hdr = reinterpret_cast<const float *>(live && in_pool ? blk : reinterpret_cast<const uint8_t *>(d.safe));
            page_sk = hdr[kvh];
            page_sv = hdr[d.Hkv + kvh];
            blk += PKV_FP8_HEADER;
        }
        blk += (size_t)kvh * 2 * TL::TILE_BYTES;
        addr_lo = (uint32_t)(uintptr_t)blk;
        addr_hi = (uint32_t)((uintptr_t)blk >> 32);
        records = live && in_pool ? 2 * TL::TILE_BYTES : 0;
    };
    int window = 1;                                       // the lanes' pages are those of pairs window .. window + 31
    auto lane_of = [&](uint32_t x, int at) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readlane((int)x, at); };
    auto tiles = [&](int k, int half) __attribute__((always_inline)) {
        const int at = 2 * (k - window) + half;
        return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<uint8_t *>(lane_of(addr_lo, at) | (uint64_t)lane_of(addr_hi, at) << 32), 0,
                                                 (int)lane_of(records, at), 0x00020000);
    };
    auto first_tiles = [&](uint32_t id, bool live, float &sk, float &sv) __attribute__((always_inline)) {
        const bool in_pool = id < d.max_block_id;
        bad |= live && !in_pool;
        live = live && in_pool;
        const uint8_t *blk = block_ptr(d, id);
        if (DT == PKV_E4M3) {
            const float *hdr = reinterpret_cast<const float *>(live ? blk : reinterpret_cast<const uint8_t *>(d.safe));
            sk = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(PKV_CONST(float, hdr)[kvh])));
            sv = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(PKV_CONST(float, hdr)[d.Hkv + kvh])));
            blk += PKV_FP8_HEADER;
        }
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(blk + (size_t)kvh * 2 * TL::TILE_BYTES), 0, live ? 2 * TL::TILE_BYTES : 0, 0x00020000);
    };
    const int voff = lane * 16;
    auto load = [&](u32x4 *r, __amdgpu_buffer_rsrc_t rsrc, int at) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < TL::NL; ++j) r[j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff + j * 1024, at, 2 /* non-temporal */);
        asm volatile("" ::: "memory");                    // in this order everywhere: loads in flight are counted
    };
    auto load_pages = [&](PairRegs<D, DT> &r, __amdgpu_buffer_rsrc_t a, __amdgpu_buffer_rsrc_t b) __attribute__((always_inline)) {
        load(r.a.k, a, 0);
        load(r.a.v, a, TL::TILE_BYTES);
        load(r.b.k, b, 0);
        load(r.b.v, b, TL::TILE_BYTES);
    };
    auto scales = [&](PairRegs<D, DT> &r, int k) __attribute__((always_inline)) {
        if (DT != PKV_E4M3) return;
        const int at = 2 * (k - window);
        r.a.sk = __uint_as_float(lane_of(__float_as_uint(page_sk), at));
        r.a.sv = __uint_as_float(lane_of(__float_as_uint(page_sv), at));
        r.b.sk = __uint_as_float(lane_of(__float_as_uint(page_sk), at + 1));
        r.b.sv = __uint_as_float(lane_of(__float_as_uint(page_sv), at + 1));
    };
    // Pair k; `more`: pair k + 1 is asked for ahead of it.  (Asked for earlier, K of pair k + 2 behind the scores and V behind the
    // products of pair k, launches took 2 to 10 % longer: 8 lognormal rows of 2048 tokens of 32/8/128 bf16 19.0, 20.0 us, 16 of 4717
    // of 10/2/128 25.3, 27.2, 30 of 366 of 40/8/128 7.7, 8.5.  Whole pages one after the other, K and V, cost 1 to 3 % less than K of
    // both and then V.)
    auto step = [&](PairRegs<D, DT> &r, PairRegs<D, DT> &o, int k, bool more) __attribute__((always_inline)) {
        if (more) {
            load_pages(o, tiles(k + 1, 0), tiles(k + 1, 1));
            scales(o, k + 1);
        }
        const int p = page0 + STEP * k;
        const int valid_a = p == n_pages - 1 ? last_valid : T;
        const int valid_b = p + 1 < pe ? (p + 1 == n_pages - 1 ? last_valid : T) : 0;
        const bool tail = valid_a < T || valid_b < T;
        const float sca = DT == PKV_E4M3 ? d.scale_log2 * r.a.sk : d.scale_log2, scb = DT == PKV_E4M3 ? d.scale_log2 * r.b.sk : d.scale_log2;
        const f32x4 sa = qk_page<D, DT>(r.a, qf), sb = qk_page<D, DT>(r.b, qf);
        float s[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[i] = sa[i] * sca;
            s[4 + i] = sb[i] * scb;
        }
        // only a row's last pair holds tokens past its context: a branch of its own, not selects in every step
        if (tail) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (4 * G + i >= valid_a) s[i] = -INFINITY;
                if (4 * G + i >= valid_b) s[4 + i] = -INFINITY;
            }
            blank_v<D, DT>(r.a.v, valid_a - 4 * G);
            blank_v<D, DT>(r.b.v, valid_b - 4 * G);
        }
        bf16x8 phv, plv;
        softmax_pair<D, DT>(st, s, r.a.sv, r.b.sv, phv, plv);
#pragma unroll
        for (int jt = 0; jt < TL::NV; ++jt) {
            const u32x2 va = v_half<D, DT>(r.a, jt), vb = v_half<D, DT>(r.b, jt);
            const bf16x8 av = as_bf16x8(mk4(va.x, va.y, vb.x, vb.y));
            st.acc[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, phv, st.acc[jt], 0, 0, 0);
            st.acc[jt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, plv, st.acc[jt], 0, 0, 0);
        }
    };
    const int n_pairs = page0 < pe ? (pe - page0 + STEP - 1) / STEP : 0;
    if (n_pairs > 0) {
        PairRegs<D, DT> ring[2];
        const __amdgpu_buffer_rsrc_t a = first_tiles(ids.a, true, ring[0].a.sk, ring[0].a.sv);
        const __amdgpu_buffer_rsrc_t b = first_tiles(ids.b, page0 + 1 < pe, ring[0].b.sk, ring[0].b.sv);
        load_pages(ring[0], a, b);
        // (The loads in flight are counted along every way the compiler sees: the loop is entered from here only, two whole steps
        // a turn with no way out between them, the odd step by itself.)
        int k = 0;
        if (n_pairs > 1) {
            locate(page0 + STEP + ahead, id);
            do {
                if (k + 2 - window >= 32) {
                    window = k + 1;
                    locate(page0 + STEP * window + ahead, id_of(page0 + STEP * window + ahead));
                }
                step(ring[0], ring[1], k, true);
                step(ring[1], ring[0], k + 1, true);
                k += 2;
            } while (k + 2 <= n_pairs);
        }
        if (k < n_pairs) step(ring[0], ring[1], k, false);
    }
    float l = st.l;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (n < g) {
        float *a = s_acc + (w * g + n) * D;
#pragma unroll
        for (int jt = 0; jt < TL::NV; ++jt) *reinterpret_cast<f32x4 *>(a + 16 * jt + 4 * G) = st.acc[jt];
        if (G == 0) {
            s_m[w * 16 + n] = st.m;
            s_l[w * 16 + n] = l;
        }
    }
    if (__any(bad) && lane == 0) atomicOr(d.err, 1u);
    __syncthreads();
    // the sums of the work-group: lane by lane four output elements of one head
    const int quads = g * (D / 4), pf = partial_floats(g, D);
    const bool whole = JOIN && n_parts == 1;
    float *mine = JOIN ? d.ws + (size_t)(seg * d.parts + part) * pf : at_part->sums;
    for (int i = threadIdx.x; i < quads; i += 64 * SMALL_WAVES) {
        const int hn = i / (D / 4), x = i - hn * (D / 4);
        float M = s_m[hn];
#pragma unroll
        for (int v = 1; v < SMALL_WAVES; ++v) M = fmaxf(M, s_m[v * 16 + hn]);
        float den = 0.f;
        f32x4 num = {0.f, 0.f, 0.f, 0.f};
        if (n_pages > 0) {                                // an empty context: the row is defined as zero
#pragma unroll
            for (int v = 0; v < SMALL_WAVES; ++v) {
                const float f = merge_weight(s_m[v * 16 + hn], M);
                den += f * s_l[v * 16 + hn];
                num += f * *reinterpret_cast<const f32x4 *>(s_acc + (v * g + hn) * D + 4 * x);
            }
        }
        if (whole) {
            *reinterpret_cast<f32x4 *>(d.out + ((size_t)seq * d.Hq + kvh * g + hn) * D + 4 * x) = n_pages > 0 && (!PREFIXED || den != 0.f) ? num * (1.0f / den) : num;
        } else {
            *reinterpret_cast<f32x4 *>(mine + hn * (JOIN ? D : D + 4) + 4 * x) = num;
            if (x == 0) {
                mine[JOIN ? g * D + hn : hn * (D + 4) + D] = M;
                mine[JOIN ? g * D + g + hn : hn * (D + 4) + D + 1] = den;
            }
        }
    }
    if (whole || !JOIN) return;
    // Hand-over as in attn_wave: partials and counters are in uncached memory, so the order of a wave's own accesses is
    // all there is to enforce; every wave's stores have landed when the counter moves.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) *s_arrived = atomicAdd(d.cnt + seg, 1u);
    __syncthreads();
    if (*s_arrived != (uint32_t)(n_parts - 1)) return;
    if (threadIdx.x == 0) d.cnt[seg] = 0u;                // ready for the next launch
    const float *base = d.ws + (size_t)seg * d.parts * pf;
    // All maxima and sums travel together with the sums of the first eight parts: one trip to uncached memory instead of two.
    // Us a launch, rows in many parts: 1 x 32000 tokens of 8/1/128 17.5 -> 15.4, 1 x 12000 of 64/8/128 14.6 -> 13.6, 3 x 6000 of
    // 28/4/128 12.6 -> 12.0, 2 x 9000 of 32/8/128 e4m3 15.7 -> 15.2; with its append 8 x 2048 of 32/8/128 16.8 -> 16.4; rows in one
    // part (4 x 128 of 8/2/64) the same.  (The read is there twice, 7 KB more over all variants.)
    auto part_sums = [&](f32x4 *v, int c0, int hn, int x) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            v[u] = *reinterpret_cast<const f32x4 *>(base + (size_t)(c0 + u < n_parts ? c0 + u : n_parts - 1) * pf + hn * D + 4 * x);
    };
    f32x4 first[8];
    {
        const int i = (int)threadIdx.x < quads ? (int)threadIdx.x : quads - 1, hn = i / (D / 4);
        part_sums(first, 0, hn, i - hn * (D / 4));
    }
    for (int i = threadIdx.x; i < n_parts * g; i += 64 * SMALL_WAVES) {
        const int c = i / g, hn = i - c * g;
        s_acc[i] = base[(size_t)c * pf + g * D + hn];
        s_acc[MAX_PIECES * 16 + i] = base[(size_t)c * pf + g * D + g + hn];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < quads; i += 64 * SMALL_WAVES) {
        const int hn = i / (D / 4), x = i - hn * (D / 4);
        float M = -INFINITY, den = 0.f;
        f32x4 num = {0.f, 0.f, 0.f, 0.f};
        for (int c = 0; c < n_parts; ++c) M = fmaxf(M, s_acc[c * g + hn]);
        for (int c0 = 0; c0 < n_parts; c0 += 8) {
            if (c0 > 0 || i >= 64 * SMALL_WAVES) part_sums(first, c0, hn, x);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (c0 + u < n_parts) {
                    const float f = PREFIXED ? merge_weight(s_acc[(c0 + u) * g + hn], M) : __builtin_amdgcn_exp2f(s_acc[(c0 + u) * g + hn] - M);
                    den += f * s_acc[MAX_PIECES * 16 + (c0 + u) * g + hn];
                    num += f * first[u];
                }
        }
        *reinterpret_cast<f32x4 *>(d.out + ((size_t)seq * d.Hq + kvh * g + hn) * D + 4 * x) = !PREFIXED || den != 0.f ? num * (1.0f / den) : num;
    }
}

}  // namespace
