// Decode attention of sequences that share prefixes (gfx950): a group's prefix is walked once, by the queries of all its members as the
// columns of one matrix product, each sequence's own row by itself, and the sums are joined.
//
//   out = (sum_i 2^(m_i - M) acc_i) / (sum_i 2^(m_i - M) l_i),  M = max_i m_i,  over the parts i of prefix and own row
//
// One launch holds both kinds of work-group: those of a prefix (prefill_unit.h: up to 128 columns of members x heads of a kv head,
// a part of the prefix, no mask: whole blocks are shared) are bound by the matrix units, those of own rows (decode_part.h: a work-group
// per part of a row) by memory, and they run side by side.  A second launch joins.
#include "decode_part.h"
#include "prefill_unit.h"

namespace {

// A group of a plan, found by one read for all lanes.
struct GroupLanes {
    uint32_t unit, first, blocks, parts, tile;
    __device__ __forceinline__ explicit GroupLanes(const PrefixPlan &plan) {
        const int i = threadIdx.x & 63;
        unit = plan.g[i].unit;
        first = plan.g[i].first;
        blocks = plan.g[i].blocks;
        parts = plan.g[i].parts;
        tile = plan.g[i].tile;
    }
    static __device__ __forceinline__ uint32_t of(uint32_t x, int i) { return (uint32_t)__builtin_amdgcn_readlane((int)x, i); }
};
static_assert(PKV_PREFIX_GROUPS == 64, "a group per lane");

struct PrefixUnit {
    static constexpr bool CAUSAL = false;
    const uint16_t *members;
    const int32_t *shared;
    int prefix_row, blocks, ntok, part, parts, tiles, first_tile;      // (tiles: of 32 columns, in the unit)

    __device__ __forceinline__ PrefixUnit(const AttnDesc &d, const PrefixPlan &plan, int unit) {
        const GroupLanes lanes(plan);
        const int n = plan.n_groups;
        // groups without units share their first unit with the next one
        const int at = __popcll(__ballot((int)(threadIdx.x & 63) < n && lanes.unit <= (uint32_t)unit)) - 1;
        const uint32_t f = lanes.of(lanes.first, at);
        const int first = (int)(f & 0xffffu), end = at + 1 < 64 ? (int)(lanes.of(lanes.first, at + 1) & 0xffffu) : (int)(plan.g[64].first & 0xffffu);
        const int tile_tok = d.cols / d.g, size = PF_WAVES * tile_tok, count = end - first, wide = (count + size - 1) / size;
        const int u = unit - (int)lanes.of(lanes.unit, at);
        part = u / wide;
        const int x = u - part * wide;
        members = plan.member + first + x * size;
        ntok = count - x * size < size ? count - x * size : size;
        blocks = (int)lanes.of(lanes.blocks, at);
        parts = (int)lanes.of(lanes.parts, at);
        prefix_row = (int)(f >> 16);
        shared = d.table + (size_t)prefix_row * d.row_stride;
        tiles = (count < size ? count + tile_tok - 1 : size) / tile_tok;
        first_tile = (int)lanes.of(lanes.tile, at) + u * d.Hkv * tiles;
    }
    __device__ __forceinline__ uint32_t id(const AttnDesc &d, int page) const { return (uint32_t)shared[page < d.row_stride ? page : d.row_stride - 1]; }
    __device__ __forceinline__ int row(int i) const { return members[i]; }
    __device__ __forceinline__ int sees(const AttnDesc &d) const {
        if (PKV_CONST(int32_t, d.row_len)[prefix_row] < blocks) {
            if (threadIdx.x == 0) atomicOr(d.err, 1u);
            return 0;
        }
        return blocks * PKV_T;
    }
    __device__ __forceinline__ bool partial() const { return true; }
    __device__ __forceinline__ size_t tile(const AttnDesc &, int kvh, int w) const { return (size_t)first_tile + kvh * tiles + w; }
};

template <int D, int DT, int MEET>
__global__ __launch_bounds__(64 * PF_WAVES, 2) void k_prefix_sums(const AttnDesc d, const PrefixPlan plan) {
    constexpr int OWN = SMALL_WAVES * 16 * D * 4 + 2 * SMALL_WAVES * 16 * 4, RING = kRingBytes<D, DT, MEET>;
    __shared__ __align__(16) uint8_t lds[OWN > RING ? OWN : RING];
    static_assert(PF_WAVES == SMALL_WAVES, "one size of work-group");
    if (blockIdx.x < plan.prefix_wgs) {
        const int unit = blockIdx.x / d.Hkv, kvh = blockIdx.x - unit * d.Hkv;
        prefill_unit<D, DT, MEET, true>(d, PrefixUnit(d, plan, unit), kvh, lds);
    } else {
        float *acc = reinterpret_cast<float *>(lds), *m = acc + SMALL_WAVES * 16 * D, *l = m + SMALL_WAVES * 16;
        attn_part<D, DT, false>(d, (int)(blockIdx.x - plan.prefix_wgs), acc, m, l, nullptr, plan.own_ws);
    }
}

// One wave per (member, query head): lane i holds the maxima and denominators of parts i and i + 64, then D / 4 lanes take the sums of a
// part, 64 * 4 / D parts side by side.  Bound by memory trips: the plan, the lengths, maxima and denominators, sums.
constexpr int JOIN_WAVES = 4;

template <int D>
__global__ __launch_bounds__(64 * JOIN_WAVES) void k_prefix_join(const AttnDesc d, const PrefixPlan plan) {
    constexpr int QUADS = D / 4, SIDE = 64 / QUADS;
    const int lane = threadIdx.x & 63;
    const int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * JOIN_WAVES + (threadIdx.x >> 6)));
    const int j = x / d.Hq, hq = x - j * d.Hq;
    if (j >= plan.n_members) return;
    const GroupLanes lanes(plan);
    const int at = __popcll(__ballot(lane < plan.n_groups && (int)(lanes.first & 0xffffu) <= j)) - 1;
    const uint32_t f = lanes.of(lanes.first, at);
    const int first = (int)(f & 0xffffu), end = at + 1 < 64 ? (int)(lanes.of(lanes.first, at + 1) & 0xffffu) : (int)(plan.g[64].first & 0xffffu);
    const int blocks = (int)lanes.of(lanes.blocks, at), parts = blocks > 0 ? (int)lanes.of(lanes.parts, at) : 0;
    const int seq = plan.member[j], kvh = hq / d.g, head = hq - kvh * d.g;
    const int L = ctx_clamped(d, seq), n_pages = (L + T - 1) / T;
    const bool missing = blocks > 0 && PKV_CONST(int32_t, d.row_len)[f >> 16] < blocks;
    // where its column is in a part of the prefix
    const int tile_tok = d.cols / d.g, size = PF_WAVES * tile_tok, count = end - first, wide = (count + size - 1) / size;
    const int tiles = (count < size ? count + tile_tok - 1 : size) / tile_tok, i = j - first, xg = i / size, in = i - xg * size, w = in / tile_tok;
    const size_t tile0 = (size_t)lanes.of(lanes.tile, at) + (size_t)(xg * d.Hkv + kvh) * tiles + w, step = (size_t)wide * d.Hkv * tiles;
    const float *prefix = d.ws + (tile0 * PF_COLS + (in - w * tile_tok) * d.g + head) * (D + 4);
    const size_t prefix_step = step * PF_COLS * (D + 4);
    // its own parts (attn_part)
    int part_pages = d.part_pages;
    if (n_pages > d.parts * part_pages) part_pages = ((n_pages + d.parts - 1) / d.parts + 2 * SMALL_WAVES - 1) / (2 * SMALL_WAVES) * (2 * SMALL_WAVES);
    const int own_parts = n_pages > part_pages ? (n_pages + part_pages - 1) / part_pages : 1;
    const int pf = partial_floats(d.g, D), all = parts + own_parts;
    const float *own = plan.own_ws + (size_t)(seq * d.Hkv + kvh) * d.parts * pf;

    float m[2], l[2], M = -INFINITY, den = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int p = lane + 64 * k;
        const float *mp = p < parts ? prefix + p * prefix_step + D : own + (size_t)(p < all ? p - parts : 0) * pf + d.g * D + head;
        m[k] = p < all ? mp[0] : -INFINITY;
        l[k] = p < all ? mp[p < parts ? 1 : d.g] : 0.f;
        M = fmaxf(M, m[k]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        m[k] = merge_weight(m[k], M);
        den += l[k] * m[k];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) den += __shfl_xor(den, o);
    const int quad = lane % QUADS, side = lane / QUADS;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < all; p0 += 8 * SIDE) {
        f32x4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            int p = p0 + SIDE * k + side;
            p = p < all ? p : all - 1;
            v[k] = *reinterpret_cast<const f32x4 *>((p < parts ? prefix + p * prefix_step : own + (size_t)(p - parts) * pf + head * D) + 4 * quad);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int p = p0 + SIDE * k + side;
            const float a = __shfl(m[0], p & 63), b = __shfl(m[1], p & 63);
            if (p < all) acc += v[k] * (p < 64 ? a : b);
        }
    }
#pragma unroll
    for (int o = QUADS; o < 64; o <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], o);
    // a row that sees nothing is defined as zero, and so is one whose prefix is not there
    const float inv = den > 0.f && !missing ? 1.0f / den : (den != den ? den : 0.f);
    if (missing) acc = f32x4{0.f, 0.f, 0.f, 0.f};
    if (side == 0) *reinterpret_cast<f32x4 *>(d.out + ((size_t)seq * d.Hq + hq) * D + 4 * quad) = acc * (missing ? 0.f : inv);
}

}  // namespace

hipError_t pkv_launch_prefix_sums(const AttnDesc &d, const PrefixPlan &plan, unsigned own_wgs, hipStream_t s) {
    static_assert(sizeof(AttnDesc) + sizeof(PrefixPlan) <= 4096, "a kernel's arguments end at 4 KB");
    static_assert(sizeof(AttnDesc) + sizeof(PlanOf<PKV_PLAN_FEW>) + sizeof(SharedRows) <= 4096, "a kernel's arguments end at 4 KB");
    const dim3 grid(plan.prefix_wgs + own_wgs), wg(64 * PF_WAVES);
    if (grid.x == 0) return hipSuccess;
    if (d.dtype == PKV_BF16) {
        if (d.D == 128) hipLaunchKernelGGL((k_prefix_sums<128, PKV_BF16, 2>), grid, wg, 0, s, d, plan);
        else hipLaunchKernelGGL((k_prefix_sums<64, PKV_BF16, 2>), grid, wg, 0, s, d, plan);
    } else {
        if (d.D == 128) hipLaunchKernelGGL((k_prefix_sums<128, PKV_E4M3, 4>), grid, wg, 0, s, d, plan);
        else hipLaunchKernelGGL((k_prefix_sums<64, PKV_E4M3, 4>), grid, wg, 0, s, d, plan);
    }
    return hipGetLastError();
}

hipError_t pkv_launch_prefix_join(const AttnDesc &d, const PrefixPlan &plan, hipStream_t s) {
    const unsigned waves = (unsigned)plan.n_members * (unsigned)d.Hq;
    if (waves == 0) return hipSuccess;
    const dim3 grid((waves + JOIN_WAVES - 1) / JOIN_WAVES), wg(64 * JOIN_WAVES);
    if (d.D == 128) hipLaunchKernelGGL(k_prefix_join<128>, grid, wg, 0, s, d, plan);
    else hipLaunchKernelGGL(k_prefix_join<64>, grid, wg, 0, s, d, plan);
    return hipGetLastError();
}
