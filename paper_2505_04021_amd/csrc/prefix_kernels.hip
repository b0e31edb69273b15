// Decode attention of sequences that share prefixes (gfx950): a group's prefix is walked once, by the queries of all its members as the
// columns of one matrix product, each sequence's own row by itself, and the sums are joined.
//
//   out = (sum_i 2^(m_i - M) acc_i) / (sum_i 2^(m_i - M) l_i),  M = max_i m_i,  over the parts i of prefix and own row
//
// One launch holds both kinds of work-group: those of a prefix (prefill_unit.h: up to 128 columns of members x heads of a kv head,
// a part of the prefix, no mask: whole blocks are shared) are bound by the matrix units, those of own rows (decode_part.h: a work-group
// per part of a row) by memory, and they run side by side.  A second launch joins.
//
// Probabilities reach the matrix unit as bf16 high and low halves, 16 significant bits, on both cache types, as those of every other decode step do:
// outputs are 2.5e-6 from 64 bits on the same inputs.  (8 bits: 1e-3.  A third part would reach fp32's own distance, some 1e-6, for a third more of the
// matrix work that bounds the walk of a prefix.)  Sums, reference points and denominators are fp32 throughout.
#include "decode_part.h"
#include "prefill_unit.h"

namespace {

// The groups of a plan and the counts of parts, one of each a lane, by one read.
struct GroupLanes {
    uint32_t unit, first, blocks, tile;
    __device__ __forceinline__ explicit GroupLanes(const PrefixPlan &plan) {
        const int i = threadIdx.x & 63;
        unit = plan.g[i].unit;
        first = plan.g[i].first;
        blocks = plan.g[i].blocks;
        tile = plan.g[i].tile;
    }
    static __device__ __forceinline__ uint32_t of(uint32_t x, int i) { return (uint32_t)__builtin_amdgcn_readlane((int)x, i); }
    __device__ __forceinline__ int first_member(const PrefixPlan &plan, int i) const {
        return (int)((i < 64 ? of(first, i) : (uint32_t)__builtin_amdgcn_readfirstlane((int)plan.g[64].first)) & 0xffffu);
    }
};
static_assert(PKV_PREFIX_GROUPS == 64 && PKV_PLAN_MAX_PARTS == 64, "one of each per lane");

// How a group's members fall into work-groups and tiles of 32 columns.
struct GroupShape {
    int size, wide, tiles;                // members of a work-group, work-groups side by side, tiles of each
    __device__ __forceinline__ GroupShape(const AttnDesc &d, int count) {
        const int tile_tok = d.cols / d.g;
        size = PF_WAVES * tile_tok;
        wide = (count + size - 1) / size;
        tiles = count < size ? (count + tile_tok - 1) / tile_tok : PF_WAVES;
    }
};

struct PrefixUnit {
    static constexpr bool CAUSAL = false, SHARED = false, MASKED = false;
    __device__ __forceinline__ int front() const { return 0; }
    // (96 rows behind 24576 tokens, without their own, in 192 work-groups 138, 146 us without levels, in 400 112.5, 115.7)
    static constexpr bool LEVELS = true;
    const PrefixPlan &plan;
    const int32_t *shared;
    int first,                            // its first member
        prefix_row, blocks, ntok, part, parts, tiles, first_tile;      // (tiles: of 32 columns, in the unit)

    // unit: among those of the wide or of the narrow groups
    __device__ __forceinline__ PrefixUnit(const AttnDesc &d, const PrefixPlan &plan, int unit, bool narrow) : plan(plan) {
        const GroupLanes lanes(plan);
        const int n = plan.n_groups;
        // the last of its kind that begins at or before it (groups without units share their first one with the next)
        const int at = 63 - __clzll((long long)__ballot((int)(threadIdx.x & 63) < n && lanes.unit <= (uint32_t)unit && (lanes.blocks >> 31 != 0) == narrow));
        const uint32_t f = lanes.of(lanes.first, at), b = lanes.of(lanes.blocks, at);
        const int first_of_group = (int)(f & 0xffffu), count = lanes.first_member(plan, at + 1) - first_of_group;
        const GroupShape shape(d, count);
        const int u = unit - (int)lanes.of(lanes.unit, at);
        part = u / shape.wide;
        const int x = u - part * shape.wide;
        first = first_of_group + x * shape.size;
        ntok = count - x * shape.size < shape.size ? count - x * shape.size : shape.size;
        blocks = (int)(b & 0xffffffu);
        parts = (int)(b >> 24 & 0x7fu);
        prefix_row = (int)(f >> 16);
        shared = d.table + (size_t)prefix_row * d.row_stride;
        tiles = shape.tiles;
        first_tile = (int)lanes.of(lanes.tile, at) + u * d.Hkv * tiles;
    }
    __device__ __forceinline__ uint32_t id(const AttnDesc &d, int page) const { return (uint32_t)shared[page < d.row_stride ? page : d.row_stride - 1]; }
    __device__ __forceinline__ int row(int i) const { return plan.member[first + i]; }
    __device__ __forceinline__ int sees(const AttnDesc &d) const {
        // (no branch around the length: it would not be the same for all lanes any more in the compiler's eyes)
        const bool missing = PKV_CONST(int32_t, d.row_len)[prefix_row] < blocks;
        if (missing && threadIdx.x == 0) atomicOr(d.err, 1u);
        return missing ? 0 : blocks * PKV_T;
    }
    __device__ __forceinline__ bool partial() const { return true; }
    __device__ __forceinline__ size_t tile(const AttnDesc &, int kvh, int w) const { return (size_t)first_tile + kvh * tiles + w; }
};

template <int D, int DT, int MEET>
__global__ __launch_bounds__(64 * PF_WAVES, 2) void k_prefix_sums(const AttnDesc d, const PrefixPlan plan) {
    constexpr int OWN = SMALL_WAVES * 16 * D * 4 + 2 * SMALL_WAVES * 16 * 4, RING = kRingBytes<D, DT, MEET>;
    __shared__ __align__(16) uint8_t lds[OWN > RING ? OWN : RING];
    static_assert(PF_WAVES == SMALL_WAVES, "one size of work-group");
    // Prefixes first: their walks are the longest.  (Own rows first: with the best number of cuts for either 64 rows behind 4096 tokens 42.2
    // and 45.8 us, 96 behind 24576 117.4 and 124.6, seven tenants on e4m3 caches 45.6 and 47.6.)
    if (blockIdx.x < plan.wide_wgs) {
        const int unit = blockIdx.x / d.Hkv, kvh = blockIdx.x - unit * d.Hkv;
        prefill_unit<D, DT, MEET, true>(d, PrefixUnit(d, plan, unit, false), kvh, lds);
        return;
    }
    RowPart at;
    if (blockIdx.x < plan.prefix_wgs) {
        const int x = (int)(blockIdx.x - plan.wide_wgs), unit = x / d.Hkv, kvh = x - unit * d.Hkv;
        const PrefixUnit u(d, plan, unit, true);
        at.seq = u.prefix_row;
        at.kvh = kvh;
        at.part = u.part;
        at.parts = u.parts;
        at.blocks = u.blocks;
        at.size = ((u.blocks + u.parts - 1) / u.parts + 2 * SMALL_WAVES - 1) / (2 * SMALL_WAVES) * (2 * SMALL_WAVES);
        at.columns = u.ntok * d.g;
        at.first = u.first;
        at.sums = d.ws + u.tile(d, kvh, 0) * PF_COLS * (D + 4);
    } else {
        const int x = (int)(blockIdx.x - plan.prefix_wgs), unit = x / d.Hkv, lane = threadIdx.x & 63;
        const uint32_t from = plan.own_unit[lane], to = plan.own_unit[lane + 1];
        at.kvh = x - unit * d.Hkv;
        at.part = __popcll(__ballot(from <= (uint32_t)unit)) - 1;
        const int rank = unit - (int)GroupLanes::of(from, at.part);
        at.parts = __popcll(__ballot(to - from > (uint32_t)rank));
        at.seq = __builtin_amdgcn_readfirstlane((int)plan.own[rank]);
        at.blocks = -1;
        at.size = d.part_pages;
        at.columns = d.g;
        at.first = 0;
        at.sums = plan.own_ws + (size_t)x * d.g * (D + 4);
    }
    float *acc = reinterpret_cast<float *>(lds), *m = acc + SMALL_WAVES * 16 * D, *l = m + SMALL_WAVES * 16;
    attn_part<D, DT, false>(d, 0, acc, m, l, nullptr, &at, plan.member);
}

// One wave per (member, query head): lane k holds the maximum and denominator of part k of the prefix and of the own row, then D / 4 lanes
// take the sums of a part, 256 / D parts side by side.  Bound by memory trips, two behind the plan: all of a row's maxima and
// denominators travel with the first sums.
constexpr int JOIN_WAVES = 4;

template <int D>
__global__ __launch_bounds__(64 * JOIN_WAVES) void k_prefix_join(const AttnDesc d, const PrefixPlan plan) {
    constexpr int QUADS = D / 4, SIDE = 64 / QUADS, TRIP = 8;
    const int lane = threadIdx.x & 63;
    const int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * JOIN_WAVES + (threadIdx.x >> 6)));
    const int j = x / d.Hq, hq = x - j * d.Hq;
    if (j >= plan.n_members) return;
    const GroupLanes lanes(plan);
    const uint32_t from = plan.own_unit[lane], to = plan.own_unit[lane + 1];
    const int seq = __builtin_amdgcn_readfirstlane((int)plan.member[j]), rank = __builtin_amdgcn_readfirstlane((int)plan.rank[j]);
    const int at = __popcll(__ballot(lane < plan.n_groups && (int)(lanes.first & 0xffffu) <= j)) - 1;
    const uint32_t f = lanes.of(lanes.first, at), b = lanes.of(lanes.blocks, at);
    const int first = (int)(f & 0xffffu), blocks = (int)(b & 0xffffffu), parts = (int)(b >> 24 & 0x7fu);
    const int kvh = hq / d.g, head = hq - kvh * d.g;
    const int there = PKV_CONST(int32_t, d.row_len)[f >> 16];
    // where its column is in a part of the prefix
    const GroupShape shape(d, lanes.first_member(plan, at + 1) - first);
    const int tile_tok = d.cols / d.g, i = j - first, xg = i / shape.size, in = i - xg * shape.size, w = in / tile_tok;
    const size_t tile0 = (size_t)lanes.of(lanes.tile, at) + (size_t)(xg * d.Hkv + kvh) * shape.tiles + w;
    const float *prefix = d.ws + (tile0 * PF_COLS + (in - w * tile_tok) * d.g + head) * (D + 4);
    const size_t prefix_step = (size_t)shape.wide * d.Hkv * shape.tiles * PF_COLS * (D + 4);
    const int own_parts = __popcll(__ballot(to - from > (uint32_t)rank)), all = parts + own_parts;
    auto own_part = [&](uint32_t k_from) __attribute__((always_inline)) {
        return plan.own_ws + (((size_t)(k_from + (uint32_t)rank) * d.Hkv + kvh) * d.g + head) * (D + 4);
    };

    float m[2], l[2];
    {
        const float *p = prefix + (lane < parts ? lane : 0) * prefix_step + D, *o = own_part(lane < own_parts ? from : lanes.of(from, 0)) + D;
        m[0] = l[0] = 0.f;
        if (parts > 0) {
            m[0] = p[0];
            l[0] = p[1];
        }
        m[1] = o[0];
        l[1] = o[1];
    }
    const int quad = lane % QUADS, side = lane / QUADS;
    f32x4 v[TRIP];
    auto sums = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < TRIP; ++k) {
            int p = p0 + SIDE * k + side;
            p = p < all ? p : all - 1;
            const uint32_t k_from = (uint32_t)__shfl((int)from, p < parts ? 0 : p - parts);
            const float *src = p < parts ? prefix + p * prefix_step : own_part(k_from);
            v[k] = *reinterpret_cast<const f32x4 *>(src + 4 * quad);
        }
    };
    sums(0);
    if (lane >= parts) {
        m[0] = -INFINITY;
        l[0] = 0.f;
    }
    if (lane >= own_parts) {
        m[1] = -INFINITY;
        l[1] = 0.f;
    }
    float M = fmaxf(m[0], m[1]), den = 0.f;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        m[k] = merge_weight(m[k], M);
        den += l[k] * m[k];                                // (a part that weighs nothing may still be NaN: it had a NaN logit, or a NaN among its values)
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) den += __shfl_xor(den, o);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < all; p0 += TRIP * SIDE) {
        if (p0 > 0) sums(p0);
#pragma unroll
        for (int k = 0; k < TRIP; ++k) {
            const int p = p0 + SIDE * k + side;
            const float a = __shfl(m[0], p & 63), c = __shfl(m[1], (p - parts) & 63), weight = p < parts ? a : (p < all ? c : 0.f);
            if (p < all) acc += v[k] * weight;
        }
    }
#pragma unroll
    for (int o = QUADS; o < 64; o <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o);
    // a row that sees nothing is defined as zero (its sums are), and so is one whose prefix is not there
    if (there < blocks) acc = f32x4{0.f, 0.f, 0.f, 0.f};
    if (den == 0.f || there < blocks) den = 1.f;
    if (side == 0) *reinterpret_cast<f32x4 *>(d.out + ((size_t)seq * d.Hq + hq) * D + 4 * quad) = acc * (1.0f / den);
}

// Small calls: a work-group per part of a whole context, prefix and all, as k_attention_small; every sequence reads the prefix for itself.
// One launch and no trip through memory where a context comes in one part.
template <int D, int DT>
__global__ __launch_bounds__(64 * SMALL_WAVES, 2) void k_attention_prefixed(const AttnDesc d, const SharedRows shared) {
    __shared__ __align__(16) float s_acc[SMALL_WAVES * 16 * 128];
    __shared__ float s_m[SMALL_WAVES * 16], s_l[SMALL_WAVES * 16];
    __shared__ uint32_t s_arrived;
    attn_part<D, DT, true, true>(d, (int)blockIdx.x, s_acc, s_m, s_l, &s_arrived, nullptr, nullptr, shared.of);
}

template <int D, int DT, int MEET>
void launch(const AttnDesc &d, const PrefixPlan &plan, hipStream_t s) {
    static_assert(sizeof(AttnDesc) + sizeof(PrefixPlan) <= 4096, "a kernel's arguments end at 4 KB");
    static_assert(sizeof(AttnDesc) + sizeof(PlanOf<PKV_PLAN_FEW>) + sizeof(SharedRows) <= 4096, "a kernel's arguments end at 4 KB");
    hipLaunchKernelGGL((k_prefix_sums<D, DT, MEET>), dim3(plan.prefix_wgs + plan.own_unit[PKV_PLAN_MAX_PARTS] * (unsigned)d.Hkv), dim3(64 * PF_WAVES), 0, s, d, plan);
    hipLaunchKernelGGL(k_prefix_join<D>, dim3(((unsigned)plan.n_members * (unsigned)d.Hq + JOIN_WAVES - 1) / JOIN_WAVES), dim3(64 * JOIN_WAVES), 0, s, d, plan);
}

}  // namespace

hipError_t pkv_launch_prefix(const AttnDesc &d, const PrefixPlan &plan, hipStream_t s) {
    if (d.dtype == PKV_BF16) {
        if (d.D == 128) launch<128, PKV_BF16, 2>(d, plan, s);
        else launch<64, PKV_BF16, 2>(d, plan, s);
    } else {
        if (d.D == 128) launch<128, PKV_E4M3, 4>(d, plan, s);
        else launch<64, PKV_E4M3, 4>(d, plan, s);
    }
    return hipGetLastError();
}

hipError_t pkv_launch_prefixed_small(const AttnDesc &d, const SharedRows &shared, hipStream_t s) {
    const dim3 grid((unsigned)(d.batch * d.Hkv * d.parts)), wg(64 * SMALL_WAVES);
    if (d.dtype == PKV_BF16) {
        if (d.D == 128) hipLaunchKernelGGL((k_attention_prefixed<128, PKV_BF16>), grid, wg, 0, s, d, shared);
        else hipLaunchKernelGGL((k_attention_prefixed<64, PKV_BF16>), grid, wg, 0, s, d, shared);
    } else {
        if (d.D == 128) hipLaunchKernelGGL((k_attention_prefixed<128, PKV_E4M3>), grid, wg, 0, s, d, shared);
        else hipLaunchKernelGGL((k_attention_prefixed<64, PKV_E4M3>), grid, wg, 0, s, d, shared);
    }
    return hipGetLastError();
}
