// How a chunk's query tokens fall into groups, one or more work-groups each (prefill_unit.h), and the join of the parts of a group's context (gfx950).
#pragma once
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

}  // namespace
