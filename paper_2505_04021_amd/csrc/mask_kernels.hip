// Attention with sliding windows and sinks, and of drafted trees, over the paged cache (gfx950).  mask_part.h says what is seen and how a
// context is walked.
#include "mask_part.h"

namespace {

// The decode step: a work-group per part of a (sequence, kv head).
template <int D, int DT>
__global__ __launch_bounds__(64 * SMALL_WAVES, 2) void k_window_decode(const AttnDesc d, const MaskArgs mk) {
    __shared__ __align__(16) float s_acc[SMALL_WAVES * 16 * 128];
    __shared__ float s_m[SMALL_WAVES * 16], s_l[SMALL_WAVES * 16];
    __shared__ uint32_t s_arrived;
    MaskUnit u;
    const int wg = blockIdx.x;
    if ((d.Hkv & 7) == 0) {                               // (as attn_part deals them)
        const int per_row = d.Hkv * d.parts, rest = wg % per_row;
        u.seq = wg / per_row;
        u.part = rest / d.Hkv;
        u.kvh = rest - u.part * d.Hkv;
    } else {
        const int n_segs = d.batch * d.Hkv, at = wg % n_segs;
        u.part = wg / n_segs;
        u.seq = at / d.Hkv;
        u.kvh = at - u.seq * d.Hkv;
    }
    u.parts = d.parts;
    u.size = d.part_pages;
    u.first = u.seq;
    u.tokens = u.chunk = 1;
    u.chunk0 = 0;
    u.slot = u.seq * d.Hkv + u.kvh;
    u.step = partial_floats(d.g, D);
    u.partial = (size_t)u.slot * u.parts * u.step;
    masked_part<D, DT, false>(d, mk, u, s_acc, s_m, s_l, nullptr, &s_arrived);
}

// Chunks and drafted trees: a unit of the plan is a group of 16 / g query tokens, or one of the parts of what it sees.
template <int D, int DT, bool TREE, int SEQS>
__global__ __launch_bounds__(64 * SMALL_WAVES, 2) void k_masked(const AttnDesc d, const MaskArgs mk, const PlanOf<SEQS> plan) {
    __shared__ __align__(16) float s_acc[SMALL_WAVES * 16 * 128];
    __shared__ float s_m[SMALL_WAVES * 16], s_l[SMALL_WAVES * 16];
    __shared__ uint32_t s_mask[TREE ? SMALL_WAVES * MASK_COLS * MASK_WORDS : 1];
    __shared__ uint32_t s_arrived;
    const PlanLanes<SEQS> lanes(plan);
    const int unit = blockIdx.x / d.Hkv, size = MASK_COLS / d.g;
    const PlanUnit pu = lanes.find(plan, (uint32_t)unit);
    MaskUnit u;
    u.seq = pu.seq;
    u.kvh = blockIdx.x - unit * d.Hkv;
    const int group = pu.unit / pu.parts;
    u.part = pu.unit - group * pu.parts;
    u.parts = pu.parts;
    u.size = d.part_pages;
    u.chunk0 = group * size;
    u.chunk = pu.rows;
    u.tokens = pu.rows - u.chunk0 < size ? pu.rows - u.chunk0 : size;
    u.first = pu.row + u.chunk0;
    u.slot = (unit - u.part) * d.Hkv + u.kvh;
    const size_t floats = partial_floats(MASK_COLS, D);
    u.partial = (size_t)u.slot * floats;
    u.step = (size_t)d.Hkv * floats;
    masked_part<D, DT, TREE>(d, mk, u, s_acc, s_m, s_l, s_mask, &s_arrived);
}

template <bool TREE, int SEQS>
void launch(const AttnDesc &d, const MaskArgs &mk, const PlanOf<SEQS> &plan, hipStream_t s) {
    static_assert(sizeof(AttnDesc) + sizeof(MaskArgs) + sizeof(plan) <= 4096, "a kernel's arguments end at 4 KB");
    const dim3 grid(plan.s[plan.n_seqs].unit * (unsigned)d.Hkv), wg(64 * SMALL_WAVES);
    if (d.dtype == PKV_BF16) {
        if (d.D == 128) hipLaunchKernelGGL((k_masked<128, PKV_BF16, TREE, SEQS>), grid, wg, 0, s, d, mk, plan);
        else hipLaunchKernelGGL((k_masked<64, PKV_BF16, TREE, SEQS>), grid, wg, 0, s, d, mk, plan);
    } else {
        if (d.D == 128) hipLaunchKernelGGL((k_masked<128, PKV_E4M3, TREE, SEQS>), grid, wg, 0, s, d, mk, plan);
        else hipLaunchKernelGGL((k_masked<64, PKV_E4M3, TREE, SEQS>), grid, wg, 0, s, d, mk, plan);
    }
}

}  // namespace

hipError_t pkv_launch_window(const AttnDesc &d, const MaskArgs &mk, hipStream_t s) {
    const dim3 grid((unsigned)(d.batch * d.Hkv * d.parts)), wg(64 * SMALL_WAVES);
    if (d.dtype == PKV_BF16) {
        if (d.D == 128) hipLaunchKernelGGL((k_window_decode<128, PKV_BF16>), grid, wg, 0, s, d, mk);
        else hipLaunchKernelGGL((k_window_decode<64, PKV_BF16>), grid, wg, 0, s, d, mk);
    } else {
        if (d.D == 128) hipLaunchKernelGGL((k_window_decode<128, PKV_E4M3>), grid, wg, 0, s, d, mk);
        else hipLaunchKernelGGL((k_window_decode<64, PKV_E4M3>), grid, wg, 0, s, d, mk);
    }
    return hipGetLastError();
}

hipError_t pkv_launch_masked(const AttnDesc &d, const MaskArgs &mk, const ChunkPlan &plan, bool tree, hipStream_t s) {
    if (plan.s[plan.n_seqs].unit == 0) return hipSuccess;
    if (plan.n_seqs <= PKV_PLAN_FEW) {
        if (tree) launch<true>(d, mk, few_of(plan), s);
        else launch<false>(d, mk, few_of(plan), s);
    } else {
        if (tree) launch<true>(d, mk, plan, s);
        else launch<false>(d, mk, plan, s);
    }
    return hipGetLastError();
}
