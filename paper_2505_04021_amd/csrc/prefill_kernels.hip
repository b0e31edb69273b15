// Chunked prefill over the shared pool (gfx950 / CDNA4): causal attention of a group of consecutive
// query tokens against the paged cache (paper Sec. 5.2).
//
// One work-group of four waves per (group, kv head).  Every wave owns a tile of 32 MFMA columns (query
// tokens x the g heads of the kv head) and walks the context a page pair (32 tokens) at a time:
//   scores   S[token][column] = K . q^T          D / 16 products 32x32x16, K as the row operand
//   output   O^T[d][column] += V^T . P           2 * D / 32 products per half of P (hi, lo)
// The accumulator layout of the first is the column-operand layout of the second once the eight tokens a
// lane holds of a page are taken as the eight contraction slots of its lane half, so probabilities never
// change lanes.  K and V tiles travel from the pool into LDS in the byte order they have in the block
// (kv_layout.h), one tile of the pair per wave.
//
// What bounds it: power, then the latency of a step.  On bf16 caches with 128-wide heads a wave's step is 24
// products (768 matrix cycles, a third of them the low half of the probabilities) and some 105 other vector
// instructions (8 more with a maximum per step instead of the sum as the sign that the reference point has to move:
// 228 -> 225 us a pass with its append, all shapes 0.7 to 1.3 % faster); by the counters of a launch a step takes a
// wave 2250 cycles, 1000 of them waiting, and the matrix units are busy 58 % of the launch at 1.85 GHz; with all
// operands zero the same kernel runs 25 % faster, and a plain 8192^3 matrix product loses as much to random data.  Why
// this shape: 32x32x16 products read half as many operand registers and LDS bytes per flop as 16x16x32, need one lane
// exchange instead of two per maximum (and that only when the reference point moves), and fill 32 columns better for
// odd g.  The step is software-pipelined by one pair: scores of pair p + 1 and the V reads of pair p are issued before
// the output products of pair p, between which the softmax of pair p + 1 runs.  The waves meet once in two pairs, four on
// e4m3 caches (every pair: 2 % slower).  8 sequences x (2048 cached + 512 new) of 32/8/128, a maximum in every step, arguments read where they are
// used and no priority levels, and with these mended: bf16 221.9, 213.3 us, e4m3 180.6, 171.8; of 32/8/64: bf16 140.1, 137.1, e4m3
// 131.2, 127.2.
#include "prefill_unit.h"

namespace {

// One unit of the launch: the query tokens of a group (rows q0 .. q0 + ntok - 1 of the packed q and out, followed by
// `back` more of the sequence's chunk) and which of `parts` parts of the context it walks.
struct GroupInfo {
    int seq, q0, ntok, back, part, parts;
};

template <int SEQS>
__device__ __forceinline__ GroupInfo group_info(const AttnDesc &d, const PlanOf<SEQS> &plan, const PlanLanes<SEQS> &lanes, int unit) {
    const PlanUnit pu = lanes.find(plan, (uint32_t)unit);
    const int size = PF_WAVES * (d.cols / d.g), groups = (pu.rows + size - 1) / size;
    const int rank = pu.parts > 1 ? pu.unit / pu.parts : pu.unit;
    const int t0 = (groups - 1 - rank) * size;
    GroupInfo g;
    g.seq = pu.seq;
    g.q0 = pu.row + t0;
    g.ntok = pu.rows - t0 < size ? pu.rows - t0 : size;
    g.back = pu.rows - t0 - g.ntok;
    g.parts = pu.parts;
    g.part = pu.unit - rank * pu.parts;
    return g;
}

// A group of a chunk's query tokens in front of its own row.
struct ChunkUnit {
    static constexpr bool CAUSAL = true, LEVELS = true, SHARED = false;
    __device__ __forceinline__ int front() const { return 0; }
    int seq, q0, ntok, back, part, parts, slot;
    const int32_t *own;
    __device__ __forceinline__ ChunkUnit(const GroupInfo &g, const AttnDesc &d, int group)
        : seq(g.seq), q0(g.q0), ntok(g.ntok), back(g.back), part(g.part), parts(g.parts), slot(group), own(d.table + (size_t)g.seq * d.row_stride) {}
    __device__ __forceinline__ uint32_t id(const AttnDesc &d, int page) const { return (uint32_t)own[page < d.row_stride ? page : d.row_stride - 1]; }
    __device__ __forceinline__ int row(int i) const { return q0 + i; }
    __device__ __forceinline__ int sees(const AttnDesc &d) const {
        int L = PKV_CONST(int32_t, d.ctx_lens)[seq];
        int cap = PKV_CONST(int32_t, d.row_len)[seq];
        asm volatile("" : "+s"(L), "+s"(cap));             // both at once
        L -= back;
        cap *= PKV_T;
        return L < 0 ? 0 : (L > cap ? cap : L);
    }
    __device__ __forceinline__ bool partial() const { return parts > 1; }
    __device__ __forceinline__ size_t tile(const AttnDesc &d, int kvh, int w) const { return ((size_t)slot * d.Hkv + kvh) * PF_WAVES + w; }
};

// The waves meet once in MEET pairs, and no wave runs further ahead than that.  An e4m3 cache leaves room in LDS for twice the
// slots that bf16 has (two work-groups a CU, three with 64-wide heads).  Us a pass, met in two and in four pairs: 8 x (2048 + 512)
// tokens of 32/8/128 179.3, 176.0; 8192 + 256 58.4, 56.5; ragged prompts 76.2, 75.1.  (Short walks: meets_often_in below.)
template <int D, int DT, int SEQS, int MEET>
__global__ __launch_bounds__(64 * PF_WAVES, 2) void k_prefill(const AttnDesc d, const PlanOf<SEQS> plan) {
    __shared__ __align__(16) uint8_t ring[kRingBytes<D, DT, MEET>];       // K slots, then V slots
    const PlanLanes<SEQS> lanes(plan);
    ask_arguments(d, plan.n_seqs, plan.seq0);
    const int group = blockIdx.x / d.Hkv, kvh = blockIdx.x - group * d.Hkv;
    // groups of a sequence come longest context first; a group of few query tokens in front of a long context comes
    // as several work-groups, each with a part of the context, that leave partial results for k_prefill_merge
    prefill_unit<D, DT, MEET, DT == PKV_BF16>(d, ChunkUnit(group_info(d, plan, lanes, group), d, group), kvh, ring);
}

// Chunks of sequences that share a prefix: the blocks of the prefix's row, then the sequence's own, as one context.  Whole blocks are
// shared, so the walk need not know where the one ends and the other begins.  Probabilities keep 16 bits on both cache types,
// so that a token's output is as exact in a chunk as in a decode step (2.5e-6 from 64 bits either way).
// On e4m3 caches with 128-wide heads the waves meet once in four pairs, also in the many short walks for which k_prefill takes two (meets_often_in
// below): us met in four and in two, 120 x 5 new tokens of 16/8/128 behind 32 12.3, 12.5, behind 128 + 32 19.7, 18.8, behind 400 + 60 32.8, 33.2; of
// 32/8/128 92 x 5 behind 64 13.5, 12.4, 120 x 20 behind 160 + 40 31.2, 31.7.
struct PrefixedUnit : ChunkUnit {
    static constexpr bool SHARED = true;
    __device__ __forceinline__ int front() const { return PKV_T * blocks; }
    const int32_t *shared;
    int seq_shared, blocks;
    __device__ __forceinline__ PrefixedUnit(const GroupInfo &g, const AttnDesc &d, int group, const SharedRow &p)
        : ChunkUnit(g, d, group), shared(d.table + (size_t)p.row * d.row_stride), seq_shared(p.row), blocks(p.blocks) {}
    __device__ __forceinline__ uint32_t id(const AttnDesc &d, int page) const {
        const int last = d.row_stride - 1, at = page < blocks ? page : page - blocks;
        return (uint32_t)(page < blocks ? shared : own)[at < last ? at : last];
    }
    __device__ __forceinline__ int sees(const AttnDesc &d) const {
        const int there = PKV_CONST(int32_t, d.row_len)[seq_shared], mine = ChunkUnit::sees(d);
        // (no branch around the length: it would not be the same for all lanes any more in the compiler's eyes)
        const bool missing = there < blocks;               // (blocks <= row_stride: the host has seen to that)
        if (missing && threadIdx.x == 0) atomicOr(d.err, 1u);
        return missing ? 0 : PKV_T * blocks + mine;
    }
};

template <int D, int DT, int MEET>
__global__ __launch_bounds__(64 * PF_WAVES, 2) void k_prefill_prefixed(const AttnDesc d, const PlanOf<PKV_PLAN_FEW> plan, const SharedRows shared) {
    __shared__ __align__(16) uint8_t ring[kRingBytes<D, DT, MEET>];
    const PlanLanes<PKV_PLAN_FEW> lanes(plan);
    ask_arguments(d, plan.n_seqs, plan.seq0);
    const int group = blockIdx.x / d.Hkv, kvh = blockIdx.x - group * d.Hkv;
    const GroupInfo gi = group_info(d, plan, lanes, group);
    prefill_unit<D, DT, MEET, true>(d, PrefixedUnit(gi, d, group, shared.of[gi.seq - plan.seq0]), kvh, ring);
}

// Joins the parts of a group whose context was walked by several work-groups of k_prefill (consecutive units):
// out = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i with M = max_i m_i, per column.  One work-group per eight
// columns, 32 lanes a column.  Bound by memory round trips: all maxima and denominators of a column travel at once,
// its sums eight parts a trip (one part after the other, 32 parts of one group took 80 of a call's 101 us).
constexpr int MERGE_COLS = 8;

template <int SEQS>
__global__ __launch_bounds__(32 * MERGE_COLS) void k_prefill_merge(const AttnDesc d, const PlanOf<SEQS> plan) {
    __shared__ float s_f[MERGE_COLS][PKV_PLAN_MAX_PARTS];
    constexpr int BLOCKS = PKV_PREFILL_COLS / MERGE_COLS;
    const int sub = threadIdx.x & 31, cc = threadIdx.x >> 5;
    const int x = blockIdx.x / BLOCKS, rank = x / d.Hkv, kvh = x - rank * d.Hkv;
    const int c = (blockIdx.x - x * BLOCKS) * MERGE_COLS + cc;
    const uint32_t entry = plan.s[blockIdx.y].unit, seq = entry >> PKV_PLAN_SEQ_SHIFT, first = plan.s[seq].row;
    const int parts = (int)(first >> PKV_PLAN_PART_SHIFT), row0 = (int)(first & PKV_PLAN_ROWS);
    const int rows = (int)(plan.s[seq + 1].row & PKV_PLAN_ROWS) - row0;
    const int tile_tok = d.cols / d.g, size = PF_WAVES * tile_tok, groups = (rows + size - 1) / size;
    if (parts <= 1 || rank >= groups) return;
    const int t0 = (groups - 1 - rank) * size;
    const int n = c & (PF_COLS - 1), tok = t0 + (c / PF_COLS) * tile_tok + n / d.g;      // this column's query token
    if (__syncthreads_or(n < d.cols && tok < rows) == 0) return;
    const int D = d.D, stride = D + 4;       // D sums, the reference point, the denominator, two unused (16-byte rows)
    const size_t step = (size_t)d.Hkv * PKV_PREFILL_COLS * stride;
    const float *part = d.ws + (((size_t)(entry & PKV_PLAN_UNITS) + (size_t)rank * parts) * d.Hkv + kvh) * PKV_PREFILL_COLS * stride + (size_t)c * stride;
    float m[2], l[2], M = PF_M0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = sub + 32 * k;
        m[k] = i < parts ? part[i * step + D] : PF_M0;
        l[k] = i < parts ? part[i * step + D + 1] : 0.f;
        M = fmaxf(M, m[k]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    float den = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = sub + 32 * k;
        const float f = i < parts ? __builtin_amdgcn_exp2f(m[k] - M) : 0.f;
        s_f[cc][i] = f;
        den += f * l[k];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) den += __shfl_xor(den, o);
    __syncthreads();
    if (n >= d.cols || tok >= rows || 4 * sub >= D) return;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < parts; i0 += 8) {
        f32x4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const f32x4 *>(part + (i0 + u < parts ? i0 + u : parts - 1) * step + 4 * sub);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i0 + u < parts) acc += v[u] * s_f[cc][i0 + u];
    }
    const float inv = den > 0.f ? 1.0f / den : 0.f;
    *reinterpret_cast<f32x4 *>(d.out + ((size_t)(row0 + tok) * d.Hq + kvh * d.g + (n - (n / d.g) * d.g)) * D + 4 * sub) = acc * inv;
}

template <int SEQS>
void launch_merge(const AttnDesc &d, const PlanOf<SEQS> &plan, int split_groups, hipStream_t s) {
    hipLaunchKernelGGL(k_prefill_merge<SEQS>, dim3((unsigned)(split_groups * d.Hkv * (PKV_PREFILL_COLS / MERGE_COLS)), (unsigned)plan.n_seqs),
                       dim3(32 * MERGE_COLS), 0, s, d, plan);
}

template <int SEQS>
void launch(const AttnDesc &d, const PlanOf<SEQS> &plan, int split_groups, bool meets_often, hipStream_t s) {
    const dim3 grid(plan.s[plan.n_seqs].unit * (unsigned)d.Hkv), wg(64 * PF_WAVES);
    if (d.dtype == PKV_BF16) {
        if (d.D == 128) hipLaunchKernelGGL((k_prefill<128, PKV_BF16, SEQS, 2>), grid, wg, 0, s, d, plan);
        else hipLaunchKernelGGL((k_prefill<64, PKV_BF16, SEQS, 2>), grid, wg, 0, s, d, plan);
    } else {
        if (d.D == 64) hipLaunchKernelGGL((k_prefill<64, PKV_E4M3, SEQS, 4>), grid, wg, 0, s, d, plan);
        else if (meets_often) hipLaunchKernelGGL((k_prefill<128, PKV_E4M3, SEQS, 2>), grid, wg, 0, s, d, plan);
        else hipLaunchKernelGGL((k_prefill<128, PKV_E4M3, SEQS, 4>), grid, wg, 0, s, d, plan);
    }
    if (split_groups > 0) launch_merge(d, plan, split_groups, s);
}

}  // namespace

// Whether the waves of an e4m3 launch with 128-wide heads meet once in two pairs.  A work-group's LDS is given back when its last wave
// ends, its registers wave by wave: with the rings for four pairs (64 KiB) a third work-group of a CU waits for the LDS, with those for
// two (32 KiB) it starts beside the last waves.  That counts where more work-groups come than two a CU and walks are short.  Us,
// met in four and in two pairs: 92 x 5 new tokens of 32/8/128 (736 work-groups of one pair) 11.0, 10.2; 128 x (176 + 5) of 16/8/128 (1024 of
// six) 22.5, 21.3.  180 launches of short chunks: one to two pairs 1.074 (513 to 768 work-groups), up to eight 1.007 to 1.026; but nine to
// sixteen 0.97 to 0.99, and within 512 work-groups 0.95 to 1.00 of any length.  64-wide heads, three a CU: 0.99 to 1.01.
static bool meets_often_in(const AttnDesc &d, const ChunkPlan &plan, int longest_walk) {
    return longest_walk <= 8 && plan.s[plan.n_seqs].unit * (unsigned)d.Hkv > 512u;
}

hipError_t pkv_launch_prefill(const AttnDesc &d, const ChunkPlan &plan, int split_groups, int longest_walk, hipStream_t s) {
    if (plan.s[plan.n_seqs].unit == 0) return hipSuccess;
    const bool meets_often = meets_often_in(d, plan, longest_walk);
    if (plan.n_seqs <= PKV_PLAN_FEW) launch(d, few_of(plan), split_groups, meets_often, s);
    else launch(d, plan, split_groups, meets_often, s);
    return hipGetLastError();
}

hipError_t pkv_launch_prefill_prefixed(const AttnDesc &d, const ChunkPlan &plan, const SharedRows &shared, int split_groups, hipStream_t s) {
    if (plan.s[plan.n_seqs].unit == 0) return hipSuccess;
    const PlanOf<PKV_PLAN_FEW> few = few_of(plan);
    const dim3 grid(few.s[few.n_seqs].unit * (unsigned)d.Hkv), wg(64 * PF_WAVES);
    if (d.dtype == PKV_BF16) {
        if (d.D == 128) hipLaunchKernelGGL((k_prefill_prefixed<128, PKV_BF16, 2>), grid, wg, 0, s, d, few, shared);
        else hipLaunchKernelGGL((k_prefill_prefixed<64, PKV_BF16, 2>), grid, wg, 0, s, d, few, shared);
    } else {
        if (d.D == 128) hipLaunchKernelGGL((k_prefill_prefixed<128, PKV_E4M3, 4>), grid, wg, 0, s, d, few, shared);
        else hipLaunchKernelGGL((k_prefill_prefixed<64, PKV_E4M3, 4>), grid, wg, 0, s, d, few, shared);
    }
    if (split_groups > 0) launch_merge(d, few, split_groups, s);
    return hipGetLastError();
}
