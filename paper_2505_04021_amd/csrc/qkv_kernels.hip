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
// frequency is held as a fraction of a circle in 64 bits and multiplied by the position modulo one circle, in integers: exact to
// 2^-32 of a circle at any position, and what v_sin_f32 and v_cos_f32 take as their argument.
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

// Eight elements e0 .. e0 + 7 of a head: factors of the element itself and of its partner (rotated elements only).
__device__ __forceinline__ void factors(const QkvArgs &a, int e0, int pos, float *cs, float *sn) {
    if (!a.turns) return;
    const int half = a.rot >> 1;
    if (a.pairs) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int pair = (e0 >> 1) + i;
            float s, c;
            turn_of(a.turns[pair < half ? pair : 0], pos, s, c);
            cs[2 * i] = cs[2 * i + 1] = c * a.magnitude;
            sn[2 * i + 1] = s * a.magnitude;
            sn[2 * i] = -sn[2 * i + 1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = e0 + i, pair = e < half ? e : (e < a.rot ? e - half : 0);
            float s, c;
            turn_of(a.turns[pair], pos, s, c);
            cs[i] = c * a.magnitude;
            sn[i] = (e < half ? -s : s) * a.magnitude;
        }
    }
}

// Eight elements turned; px: their partners, of the half layout only.
__device__ __forceinline__ void turn8(const QkvArgs &a, int e0, float *x, const float *px, const float *cs, const float *sn) {
    if (!a.turns) return;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * cs[i] + (a.pairs ? x[i ^ 1] : px[i]) * sn[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = e0 + i < a.rot ? y[i] : x[i];
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

// The keys of a page on their way into its tile (kv_pages.h).  pos: the position of slot 0's token.
template <int D>
struct TurnKeys {
    const QkvArgs &a;
    const int pos0;
    int t, c;
    uint32_t px[D / 32][4];                               // the partners of this lane's elements, half layout

    __device__ __forceinline__ TurnKeys(const QkvArgs &args, int pos) : a(args), pos0(pos) {}

    __device__ __forceinline__ void ask(const PageRows &p, int slot, int col) {
        t = slot;
        c = col;
        const int half = a.rot >> 1;
        if (!a.turns || a.pairs) {
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) px[j][i] = 0u;
        } else if (p.aligned && (half & 7) == 0) {
#pragma unroll
            for (int j = 0; j < D / 32; ++j) row_bytes<16, 2, true>(px[j], p, t, 2 * partner_of(a, 8 * (4 * j + c)));
        } else {
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t w[1];
                    const int at = partner_of(a, 8 * (4 * j + c) + i);
                    row_bytes<4, 2, false>(w, p, t, 2 * (at & ~1));
                    const uint32_t b = (at & 1) ? w[0] >> 16 : w[0] & 0xffffu;
                    px[j][i >> 1] = (i & 1) ? px[j][i >> 1] | b << 16 : b;
                }
        }
    }

    __device__ __forceinline__ void turn(uint32_t *words) {
        float r = 1.f;
        if (a.k_weight) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                float x[8];
                widen(x, words + 4 * j);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
            }
            r = 1.0f / sqrtf(lanes4_sum(sum) * (1.0f / D) + a.eps);
        }
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const int e0 = 8 * (4 * j + c);
            float x[8], p[8], cs[8], sn[8];
            widen(x, words + 4 * j);
            widen(p, px[j]);
            if (a.k_weight) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] *= r * bf16_of(a.k_weight[e0 + i]);
                    p[i] *= r * bf16_of(a.k_weight[partner_of(a, e0 + i)]);
                }
            }
            factors(a, e0, pos0 + t, cs, sn);
            turn8(a, e0, x, p, cs, sn);
#pragma unroll
            for (int i = 0; i < 4; ++i) words[4 * j + i] = pack_bf16_rne(x[2 * i], x[2 * i + 1]);
        }
    }
};

struct TurnKeysOf {
    const QkvArgs &a;
    int pos;
    template <int D>
    __device__ __forceinline__ TurnKeys<D> of() const { return TurnKeys<D>(a, pos); }
};

// Heads head0 .. head0 + heads - 1 of one token's query, 8 elements a lane, 64 * 8 / D heads at a time: read, normed, turned and written
// as whole rows of 16-byte pieces.  The angles are worked out once for all heads.
template <int D>
__device__ __forceinline__ void turn_queries(const AttnDesc &d, const QkvArgs &a, int64_t row, int pos, int head0, int heads) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES;
    const int lane = threadIdx.x & 63, c = lane % LANES, e0 = 8 * c, half = a.rot >> 1;
    const bool halves = a.turns && !a.pairs, whole = a.q_aligned && (half & 7) == 0;
    float cs[8], sn[8], w[8], pw[8];
    factors(a, e0, pos, cs, sn);
    if (a.q_weight) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = bf16_of(a.q_weight[e0 + i]);
            pw[i] = bf16_of(a.q_weight[partner_of(a, e0 + i)]);
        }
    }
    const int from = lane - c + (halves ? partner_of(a, e0) >> 3 : c);       // where whole partners are
    const uint16_t *src = a.q + row * a.q_stride;
    uint16_t *dst = a.q_out + row * d.Hq * D;
    for (int h0 = head0; h0 < head0 + heads; h0 += ROWS) {
        const int h = h0 + lane / LANES;
        const bool live = h < head0 + heads;
        const uint16_t *x_at = src + (live ? h : head0) * D;
        uint32_t xw[4], pxw[4];
        if (a.q_aligned) {
            const u32x4 v = *reinterpret_cast<const u32x4 *>(x_at + e0);
#pragma unroll
            for (int i = 0; i < 4; ++i) xw[i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) xw[i] = x_at[e0 + 2 * i] | (uint32_t)x_at[e0 + 2 * i + 1] << 16;
        }
        if (halves && whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) pxw[i] = (uint32_t)__shfl((int)xw[i], from);
        } else if (halves) {
#pragma unroll
            for (int i = 0; i < 4; ++i) pxw[i] = x_at[partner_of(a, e0 + 2 * i)] | (uint32_t)x_at[partner_of(a, e0 + 2 * i + 1)] << 16;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) pxw[i] = 0u;
        }
        float x[8], p[8];
        widen(x, xw);
        widen(p, pxw);
        if (a.q_weight) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
            const float r = 1.0f / sqrtf(head_sum<LANES>(sum) * (1.0f / D) + a.eps);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                x[i] *= r * w[i];
                p[i] *= r * pw[i];
            }
        }
        turn8(a, e0, x, p, cs, sn);
        if (live)
            *reinterpret_cast<u32x4 *>(dst + h * D + e0) =
                mk4(pack_bf16_rne(x[0], x[1]), pack_bf16_rne(x[2], x[3]), pack_bf16_rne(x[4], x[5]), pack_bf16_rne(x[6], x[7]));
    }
}

__device__ __forceinline__ void turn_queries(const AttnDesc &d, const QkvArgs &a, int64_t row, int pos, int head0) {
    const int heads = d.Hq - head0 < a.wave_heads ? d.Hq - head0 : a.wave_heads;
    if (d.D == 128) turn_queries<128>(d, a, row, pos, head0, heads);
    else turn_queries<64>(d, a, row, pos, head0, heads);
}

// The decode step.  One wave per (sequence, kv head) for K and V of its new token, the element layout of k_kv_append, then
// waves for the queries.  Bound by dependent memory trips (context length, block id, the block).
template <int DT>
__global__ __launch_bounds__(64) void k_qkv_append(const AttnDesc d, const QkvArgs a) {
    const int lane = threadIdx.x, D = d.D, kv_waves = d.batch * d.Hkv;
    if ((int)blockIdx.x >= kv_waves) {
        const int x = blockIdx.x - kv_waves, per = (d.Hq + a.wave_heads - 1) / a.wave_heads, seq = x / per;
        const int before = a.before ? PKV_CONST(int32_t, a.before)[seq] : 0;
        turn_queries(d, a, seq, before + PKV_CONST(int32_t, d.ctx_lens)[seq] - 1, (x - seq * per) * a.wave_heads);
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
    {
        float x[2] = {bf16_lo(kx[0]), bf16_lo(kx[1])}, p[2] = {bf16_lo(kp[0]), bf16_lo(kp[1])};
        float r = 1.f;
        if (a.k_weight) {
            float sum = x[0] * x[0] + (D > 64 ? x[1] * x[1] : 0.f);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            r = 1.0f / sqrtf(sum / (float)D + a.eps);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = i ? second : lane, pe = partner_of(a, e), half = a.rot >> 1;
            if (a.k_weight) {
                x[i] *= r * bf16_of(a.k_weight[e]);
                p[i] *= r * bf16_of(a.k_weight[pe]);
            }
            if (a.turns && e < a.rot) {
                const int pair = a.pairs ? e >> 1 : (e < half ? e : e - half);
                float s, c;
                turn_of(a.turns[pair], before + ctx - 1, s, c);
                x[i] = x[i] * (c * a.magnitude) + p[i] * ((e < pe ? -s : s) * a.magnitude);
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

// A prefill chunk.  Waves of whole pages as in k_kv_append_chunk (one per page the chunk touches, kv head, and K or V), then waves for
// the queries, each with some heads of one token.
constexpr int QKV_WAVES = 4;

template <int DT, int SEQS>
__global__ __launch_bounds__(64 * QKV_WAVES) void k_qkv_append_chunk(const AttnDesc d, const QkvArgs a, const PlanOf<SEQS> plan) {
    const int lane = threadIdx.x & 63;
    const PlanLanes<SEQS> lanes(plan);
    const int n_seqs = plan.n_seqs;
    int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * QKV_WAVES + (threadIdx.x >> 6)));
    const int kv_waves = (int)lanes.units(plan) * d.Hkv * 2;
    if (x >= kv_waves) {
        x -= kv_waves;
        const int per = (d.Hq + a.wave_heads - 1) / a.wave_heads, row0 = (int)(lanes.pick(lanes.row, 0) & PKV_PLAN_ROWS);
        const int row = row0 + x / per;
        if (row >= (int)(lanes.pick(lanes.row, n_seqs) & PKV_PLAN_ROWS)) return;           // the last work-group may have waves to spare
        const PlanUnit pu = lanes.find_row(plan, (uint32_t)row);
        const int before = a.before ? PKV_CONST(int32_t, a.before)[pu.seq] : 0, ctx = PKV_CONST(int32_t, d.ctx_lens)[pu.seq];
        turn_queries(d, a, row, before + ctx - pu.rows + row - pu.row, (x % per) * a.wave_heads);
        return;
    }
    const int which = x & 1, hp = x >> 1, unit = hp / d.Hkv, h = hp - unit * d.Hkv;
    const PlanUnit pu = lanes.find(plan, (uint32_t)unit);
    const int ctx = PKV_CONST(int32_t, d.ctx_lens)[pu.seq], cap = PKV_CONST(int32_t, d.row_len)[pu.seq] * PKV_T;
    const int before = a.before ? PKV_CONST(int32_t, a.before)[pu.seq] : 0;
    if ((ctx < pu.rows) | (ctx < 1) | (ctx > cap)) {
        if (lane == 0) atomicOr(d.err, 2u);
        return;
    }
    const int tok0 = ctx - pu.rows, page = tok0 / PKV_T + pu.unit;
    const int lo = tok0 > page * PKV_T ? tok0 : page * PKV_T, hi = ctx < (page + 1) * PKV_T ? ctx : (page + 1) * PKV_T;
    if (lo >= hi) return;
    const uint32_t id = (uint32_t)PKV_CONST(int32_t, d.table)[(size_t)pu.seq * d.row_stride + page];
    const uint16_t *src = which ? a.v : a.k;
    const int64_t stride = which ? a.v_stride : a.k_stride;
    PageRows p;
    p.stride = (size_t)stride * 2;
    p.src = reinterpret_cast<const uint8_t *>(src + (pu.row + (lo - tok0)) * stride + (size_t)h * d.D);
    p.s0 = lo % PKV_T;
    p.n = hi - lo;
    p.aligned = ((reinterpret_cast<uintptr_t>(src) | (uintptr_t)(stride * 2)) & 15) == 0;
    page_tile<DT, true>(d, [&]() __attribute__((always_inline)) -> uint8_t * {
        if (id >= d.max_block_id) {
            if (lane == 0) atomicOr(d.err, 1u);
            return nullptr;
        }
        return block_ptr(d, id);
    }, h, which, p, TurnKeysOf{a, before + page * PKV_T});
}

}  // namespace

hipError_t pkv_launch_qkv_append(const AttnDesc &d, const QkvArgs &a, hipStream_t s) {
    const unsigned waves = (unsigned)d.batch * (unsigned)(d.Hkv + (d.Hq + a.wave_heads - 1) / a.wave_heads);
    if (waves == 0) return hipSuccess;
    if (d.dtype == PKV_BF16) hipLaunchKernelGGL(k_qkv_append<PKV_BF16>, dim3(waves), dim3(64), 0, s, d, a);
    else hipLaunchKernelGGL(k_qkv_append<PKV_E4M3>, dim3(waves), dim3(64), 0, s, d, a);
    return hipGetLastError();
}

template <int SEQS>
static void launch_chunk(const AttnDesc &d, const QkvArgs &a, const PlanOf<SEQS> &plan, dim3 grid, hipStream_t s) {
    static_assert(sizeof(AttnDesc) + sizeof(QkvArgs) + sizeof(PlanOf<SEQS>) <= 4096, "a kernel's arguments end at 4 KB");
    if (d.dtype == PKV_BF16) hipLaunchKernelGGL((k_qkv_append_chunk<PKV_BF16, SEQS>), grid, dim3(64 * QKV_WAVES), 0, s, d, a, plan);
    else hipLaunchKernelGGL((k_qkv_append_chunk<PKV_E4M3, SEQS>), grid, dim3(64 * QKV_WAVES), 0, s, d, a, plan);
}

hipError_t pkv_launch_qkv_append_chunk(const AttnDesc &d, const QkvArgs &a, const ChunkPlan &plan, hipStream_t s) {
    const uint64_t rows = (plan.s[plan.n_seqs].row & PKV_PLAN_ROWS) - (plan.s[0].row & PKV_PLAN_ROWS);
    const uint64_t waves = (uint64_t)plan.s[plan.n_seqs].unit * d.Hkv * 2 + rows * ((d.Hq + a.wave_heads - 1) / a.wave_heads);
    if (rows == 0) return hipSuccess;
    if (waves > 0x7fffffffu) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)((waves + QKV_WAVES - 1) / QKV_WAVES));
    if (plan.n_seqs <= PKV_PLAN_FEW) launch_chunk(d, a, few_of(plan), grid, s);
    else launch_chunk(d, a, plan, grid, s);
    return hipGetLastError();
}
