// Drafted tokens that stay (gfx950): those of an accepted path are moved together behind the context, in the blocks of the paged cache, for all
// layers of a model in one launch.
//
//   token base + j becomes what token base + kept[j] was,  kept[0] < kept[1] < ...
//
// A wave per (sequence, layer, kv head, K or V) walks the pages that tokens move to: it reads the up to 16 tokens that go into one, then writes
// them.  Since kept[j] >= j, what a page receives comes from that page or later ones, which are still as they were: neither the order
// of the waves nor that of the pages matters beyond that.  An e4m3 block has one scale: a token that moves is decoded, rounded to bf16 once and appended under
// the running scale of the block it comes to, as kv_gather and kv_append would do it; tokens at the front that are in their place already
// keep their codes.
//
// Bound by dependent trips (lengths and path, block ids, tokens): the paths of four chats of 8/2/64 2.4 us; of 32 sequences with 26 drafts, eight layers of
// 32/8/128, 3.8 MB written, 7.9 us.
#include "kv_pages.h"

namespace {

constexpr int KEEP_WAVES = 4;

template <int D, int DT, bool IS_V>
__device__ __forceinline__ void move_tokens(const AttnDesc &d, const uint8_t *pool, const int32_t *row, int h, int base, const int32_t *kept, int from, int n) {
    constexpr int E = DT == PKV_BF16 ? 2 : 1, TILE = PKV_T * D * E;
    const int lane = threadIdx.x & 63, t = lane & 15, c = lane >> 4, G = t >> 2, e = t & 3;
    const size_t offset = (DT == PKV_E4M3 ? PKV_FP8_HEADER : 0) + ((size_t)h * 2 + (IS_V ? 1 : 0)) * TILE;
    auto block = [&](int page) __attribute__((always_inline)) -> uint8_t * {
        const uint32_t id = (uint32_t)row[page];
        if (id >= d.max_block_id) {
            atomicOr(d.err, 1u);
            return nullptr;
        }
        const uint32_t f = fastdiv_div(id, d.slots_div);
        return const_cast<uint8_t *>(pool) + (uint64_t)f * d.frame_bytes + (uint64_t)(id - f * d.slots_div.d) * d.block_bytes;
    };
    for (int page = (base + from) / PKV_T; page * PKV_T < base + n; ++page) {
        const int lo = base + from > page * PKV_T ? base + from : page * PKV_T, hi = base + n < (page + 1) * PKV_T ? base + n : (page + 1) * PKV_T;
        const int s0 = lo - page * PKV_T, end = hi - page * PKV_T;
        // the token that comes to this lane's slot (a slot that receives none takes the nearest that does: it is not stored)
        const int slot = t < s0 ? s0 : (t < end ? t : end - 1);
        const int src = base + kept[page * PKV_T + slot - base], ts = src % PKV_T;
        const uint8_t *blk = block(src / PKV_T);
        const uint8_t *tile = blk ? blk + offset : reinterpret_cast<const uint8_t *>(d.safe);
        if constexpr (DT == PKV_BF16) {
            u32x4 k[D / 32];
            uint32_t w[D / 32][4];
            if constexpr (!IS_V) {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) k[i] = *reinterpret_cast<const u32x4 *>(tile + ((4 * i + c) * 16 + ts) * 16);
            } else {
                // elements 32 i + 4 c .. + 3 and 32 i + 16 + 4 c .. + 3 of token ts
                const uint16_t *v = reinterpret_cast<const uint16_t *>(tile) + ((ts >> 2) * 16 + 4 * c) * 8 + (ts & 3);
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t x = v[i * 512 + r * 8 + half * 4];
                            uint32_t &to = w[i][2 * half + (r >> 1)];
                            to = r & 1 ? to | x << 16 : x;
                        }
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // all read before anything is written
            uint8_t *out = block(page);
            if (!out) continue;
            out += offset;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                if constexpr (!IS_V) {
                    if (t >= s0 && t < end) *reinterpret_cast<u32x4 *>(out + ((4 * i + c) * 16 + t) * 16) = k[i];
                } else {
                    const u32x2 a = transpose_halves(w[i][0], w[i][1], e), b = transpose_halves(w[i][2], w[i][3], e);
                    put_v_unit<2>(out + ((i * 4 + G) * 16 + 4 * c + e) * 16, mk4(a.x, a.y, b.x, b.y), G, s0, end);
                }
            }
        } else {
            const float scale = blk ? reinterpret_cast<const float *>(blk)[(IS_V ? d.Hkv : 0) + h] : 0.f;
            uint32_t x[D / 8];
            auto values = [&](uint32_t *to, uint32_t codes) __attribute__((always_inline)) {
                const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
                to[0] = pack_bf16_rne(a[0] * scale, a[1] * scale);
                to[1] = pack_bf16_rne(b[0] * scale, b[1] * scale);
            };
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                if constexpr (!IS_V) {
                    const u32x4 u = *reinterpret_cast<const u32x4 *>(tile + ((i * 4 + c) * 16 + ts) * 16);
#pragma unroll
                    for (int k = 0; k < 4; ++k) values(x + 8 * i + 2 * k, u[k]);
                } else {
                    u32x4 u[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) u[r] = *reinterpret_cast<const u32x4 *>(tile + ((i * 4 + (ts >> 2)) * 16 + 4 * c + r) * 16);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t codes = 0u;
#pragma unroll
                        for (int r = 0; r < 4; ++r) codes |= (u[r][k] >> (8 * (ts & 3)) & 0xffu) << (8 * r);
                        values(x + 8 * i + 2 * k, codes);
                    }
                }
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            quantise_values<D, IS_V>(x, [&](float *&scale_p) __attribute__((always_inline)) -> uint8_t * {
                uint8_t *out = block(page);
                scale_p = reinterpret_cast<float *>(out) + (IS_V ? d.Hkv : 0) + h;
                return out ? out + offset : out;
            }, s0, end, [] {});
        }
    }
}

template <int DT>
__global__ __launch_bounds__(64 * KEEP_WAVES) void k_kv_keep(const AttnDesc d, const ChunkPlan plan, int layers, size_t layer_bytes, const int32_t *kept,
                                                             const int32_t *n_kept, int32_t *new_lens) {
    const int lane = threadIdx.x & 63, i = blockIdx.y, seq = plan.seq0 + i;
    const int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * KEEP_WAVES + (threadIdx.x >> 6)));
    const int which = x & 1, rest = x >> 1, layer = rest / d.Hkv, h = rest - layer * d.Hkv;
    if (layer >= layers) return;                          // the last work-group may have waves to spare
    const int row0 = (int)(plan.s[i].row & PKV_PLAN_ROWS), drafted = (int)(plan.s[i + 1].row & PKV_PLAN_ROWS) - row0;
    const int ctx = PKV_CONST(int32_t, d.ctx_lens)[seq], n = PKV_CONST(int32_t, n_kept)[seq], cap = PKV_CONST(int32_t, d.row_len)[seq] * PKV_T;
    kept += row0;
    int at = lane < drafted ? kept[lane] : 0;             // (asked for with the lengths)
    const int base = ctx - drafted;
    bool fine = base >= 0 && ctx <= cap && n >= 0 && n <= drafted;
    int from = n;                                         // the first token that is not in its place already
    if (fine) {
        int front = -1;
        for (int j0 = 0; j0 < n; j0 += 64) {
            const int j = j0 + lane;
            if (j0 > 0) at = j < n ? kept[j] : 0;
            int last = __shfl_up(at, 1);
            if (lane == 0) last = front;
            front = __builtin_amdgcn_readlane(at, 63);
            if (__any(j < n && (at <= last || at >= drafted))) fine = false;
            const uint64_t moves = __ballot(j < n && at != j);
            if (moves && from == n) from = j0 + (int)__ffsll((long long)moves) - 1;
        }
    }
    if (x == 0 && lane == 0) {
        if (!fine) atomicOr(d.err, 2u);
        if (new_lens) new_lens[seq] = fine ? base + n : ctx;
    }
    if (!fine || from == n) return;
    const uint8_t *pool = d.pool_base + (size_t)layer * layer_bytes;
    const int32_t *row = d.table + (size_t)seq * d.row_stride;
    if (d.D == 128) {
        if (which) move_tokens<128, DT, true>(d, pool, row, h, base, kept, from, n);
        else move_tokens<128, DT, false>(d, pool, row, h, base, kept, from, n);
    } else {
        if (which) move_tokens<64, DT, true>(d, pool, row, h, base, kept, from, n);
        else move_tokens<64, DT, false>(d, pool, row, h, base, kept, from, n);
    }
}

}  // namespace

hipError_t pkv_launch_kv_keep(const AttnDesc &d, const ChunkPlan &plan, int layers, size_t layer_bytes, const int32_t *kept, const int32_t *n_kept,
                              int32_t *new_lens, hipStream_t s) {
    static_assert(sizeof(AttnDesc) + sizeof(ChunkPlan) + 40 <= 4096, "a kernel's arguments end at 4 KB");
    if (plan.n_seqs == 0) return hipSuccess;
    const unsigned waves = (unsigned)layers * (unsigned)d.Hkv * 2u;
    const dim3 grid((waves + KEEP_WAVES - 1) / KEEP_WAVES, (unsigned)plan.n_seqs), wg(64 * KEEP_WAVES);
    if (d.dtype == PKV_BF16) hipLaunchKernelGGL(k_kv_keep<PKV_BF16>, grid, wg, 0, s, d, plan, layers, layer_bytes, kept, n_kept, new_lens);
    else hipLaunchKernelGGL(k_kv_keep<PKV_E4M3>, grid, wg, 0, s, d, plan, layers, layer_bytes, kept, n_kept, new_lens);
    return hipGetLastError();
}
