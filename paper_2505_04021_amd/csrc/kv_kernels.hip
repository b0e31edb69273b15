// The write path of the shared pool (gfx950): bulk fill, the decode step's append of one
// new token per sequence, and a read-back in the logical layout.
//
// Paper: Sec. 4.2, D2 — a growing sequence takes its next token block from the slots of
// its model's pages; these kernels put K and V of the new tokens into that block, in the
// operand order the attention kernels read (kv_layout.h).
#include "kv_pages.h"

namespace {

// kv_read: the inverse gather, plus the scale of each token's block.
template <int DT>
__global__ void k_kv_read(AttnDesc d, const int32_t *row, int tok_begin, int n_tok, uint8_t *k, uint8_t *v, float *ks,
                          float *vs) {
    constexpr int E = DT == PKV_BF16 ? 2 : 1;
    const int D = d.D, Hkv = d.Hkv;
    const int64_t total = (int64_t)n_tok * Hkv * D;
    const int64_t idx = blockIdx.x * (int64_t)blockDim.x + threadIdx.x;
    if (idx >= total) return;
    const int dd = (int)(idx % D);
    const int h = (int)((idx / D) % Hkv);
    const int ti = (int)(idx / ((int64_t)D * Hkv));
    const int tok = tok_begin + ti;
    const int page = tok / PKV_T, t = tok % PKV_T;
    const uint8_t *blk = block_ptr(d, (uint32_t)row[page]);
    if (DT == PKV_E4M3) {
        if (dd == 0) {
            ks[(size_t)ti * Hkv + h] = reinterpret_cast<const float *>(blk)[h];
            vs[(size_t)ti * Hkv + h] = reinterpret_cast<const float *>(blk)[Hkv + h];
        }
        blk += PKV_FP8_HEADER;
    }
    const size_t tile = (size_t)PKV_T * D * E;
    const uint8_t *kt = blk + (size_t)h * 2 * tile, *vt = kt + tile;
    if (DT == PKV_BF16) {
        reinterpret_cast<uint16_t *>(k)[idx] = reinterpret_cast<const uint16_t *>(kt)[k_elem_off<DT>(t, dd)];
        reinterpret_cast<uint16_t *>(v)[idx] = reinterpret_cast<const uint16_t *>(vt)[v_elem_off<DT>(t, dd)];
    } else {
        k[idx] = kt[k_elem_off<DT>(t, dd)];
        v[idx] = vt[v_elem_off<DT>(t, dd)];
    }
}

constexpr int PAGE_WAVES = 4;       // waves of a work-group; wave x of the launch: K or V, kv head, page, fastest first

// kv_write: logical [n_tok][Hkv][D] values (bf16) or codes with their scales (e4m3) -> the in-block operand layouts.
// Rows first, then the block: us a launch on 8 x 128 heads, element loops that wait for the block first and now: one token 3.3 ->
// 2.6 bf16, 3.3 -> 2.4 e4m3, 8192 bf16 tokens 11.8 -> 12.0, 16000 21.0 -> 21.5, 32000 49.7 -> 39.6.  All arguments at once pay off
// for bf16 and for few e4m3 tokens (0.1 us), but cost many e4m3 tokens more than they had gained: 8192 10.0 and 9.6 without, 12000 14.1
// and 12.5 (13.0 before), 32000 28.5 and 26.8.
template <int DT>
__global__ __launch_bounds__(64 * PAGE_WAVES) void k_kv_write(const AttnDesc d, const int32_t *row, int tok_begin, int n_tok,
                                                              const uint8_t *k, const uint8_t *v, const float *ks, const float *vs) {
    constexpr int E = DT == PKV_BF16 ? 2 : 1;
    if constexpr (DT == PKV_BF16) {                        // (e4m3: see above)
        ask_arguments(d, k, v);
        asm volatile("" ::"s"(row), "s"(tok_begin), "s"(n_tok));
    }
    const int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * PAGE_WAVES + (threadIdx.x >> 6)));
    const int which = x & 1, hp = x >> 1, j = hp / d.Hkv, h = hp - j * d.Hkv;
    const int page = tok_begin / PKV_T + j, end = tok_begin + n_tok;
    const int lo = page * PKV_T > tok_begin ? page * PKV_T : tok_begin, hi = (page + 1) * PKV_T < end ? (page + 1) * PKV_T : end;
    if (lo >= hi) return;
    const uint32_t id = (uint32_t)PKV_CONST(int32_t, row)[page];
    const uint8_t *src = which ? v : k;
    PageRows p;
    p.stride = (size_t)d.Hkv * d.D * E;
    p.src = src + (size_t)(lo - tok_begin) * p.stride + (size_t)h * d.D * E;
    p.s0 = lo % PKV_T;
    p.n = hi - lo;
    p.aligned = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
    float scale = 0.f;
    if (DT == PKV_E4M3) scale = (which ? vs : ks)[(size_t)j * d.Hkv + h];
    page_tile<DT, false>(d, [&]() __attribute__((always_inline)) {
        uint8_t *blk = block_ptr(d, id);
        if (DT == PKV_E4M3 && (threadIdx.x & 63) == 0) reinterpret_cast<float *>(blk)[(which ? d.Hkv : 0) + h] = scale;
        return blk;
    }, h, which, p);
}

// kv_append, the decode step: one wave per (sequence, kv head) writes the token with index ctx_lens[seq] - 1 from row
// `seq` of k_new / v_new (bf16 [batch][Hkv][D]).  A context length outside what the row holds is skipped and reported
// through the device error flags (bit 1).
template <int DT>
__global__ __launch_bounds__(64) void k_kv_append(const AttnDesc d, const uint16_t *k_new, const uint16_t *v_new) {
    const int lane = threadIdx.x;
    ask_arguments(d, k_new, v_new);
    const int seq = blockIdx.x / d.Hkv, h = blockIdx.x - seq * d.Hkv;
    const int D = d.D;
    // The new token's values are asked for along with the context length: the launch is bound by its dependent memory
    // trips (context length, block id, the block), not by what it moves.
    const size_t src = ((size_t)seq * d.Hkv + h) * D + lane;
    const size_t second = src + (D > 64 ? 64 : 0);         // (no branch: it would wait for the first loads)
    uint32_t kx[2] = {k_new[src], k_new[second]}, vx[2] = {v_new[src], v_new[second]};
    asm volatile("" ::: "memory");                         // issued here: the compiler would put them where they are used
    const int ctx = PKV_CONST(int32_t, d.ctx_lens)[seq];
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

// kv_append_chunk: the sequence's new tokens, at indices ctx_lens[seq] - tokens .. ctx_lens[seq] - 1, come from
// consecutive rows, each written exactly as a single append would; one wave per (sequence, j-th page the chunk touches,
// kv head, K or V).  Where the chunk starts is known only here (ctx_lens is device data), so the plan has one page more
// than the chunk can touch and a wave whose page holds none of the chunk leaves.  Tokens of one page go in order (the
// e4m3 scale rule is sequential within a block by definition); pages do not depend on each other (a block's scale
// starts afresh at its first slot).
template <int DT, int SEQS>
__global__ __launch_bounds__(64 * PAGE_WAVES) void k_kv_append_chunk(const AttnDesc d, const PlanOf<SEQS> plan, const uint16_t *k_new,
                                                                     const uint16_t *v_new) {
    const int lane = threadIdx.x & 63;
    const PlanLanes<SEQS> lanes(plan);
    ask_arguments(d, k_new, v_new);
    asm volatile("" ::"s"(plan.n_seqs), "s"(plan.seq0));
    const int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * PAGE_WAVES + (threadIdx.x >> 6)));
    const int which = x & 1, hp = x >> 1, unit = hp / d.Hkv, h = hp - unit * d.Hkv;
    if ((uint32_t)unit >= lanes.units(plan)) return;                 // the last work-group may have waves to spare
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
    const uint16_t *src = which ? v_new : k_new;
    PageRows p;
    p.stride = (size_t)d.Hkv * d.D * 2;
    p.src = reinterpret_cast<const uint8_t *>(src) + (size_t)(pu.row + (lo - tok0)) * p.stride + (size_t)h * d.D * 2;
    p.s0 = lo % PKV_T;
    p.n = hi - lo;
    p.aligned = (reinterpret_cast<uintptr_t>(src) & 15) == 0;
    page_tile<DT, true>(d, [&]() __attribute__((always_inline)) -> uint8_t * {
        if (id >= d.max_block_id) {
            if (lane == 0) atomicOr(d.err, 1u);
            return nullptr;
        }
        return block_ptr(d, id);
    }, h, which, p);
}

// kv_gather: cached tokens of several sequences as packed bf16 rows, the way back of kv_append_chunk.  One wave per (sequence, page its
// range touches, kv head, K or V): whole 16-byte units are read, 1 KiB a request, V units are transposed between the wave's rows of 16
// lanes, and every lane stores pieces of 16 bytes, a quad's four side by side.  Codes are decoded, multiplied by their block's scale in fp32
// and rounded to bf16 once.  Bound by memory, every byte once, and for short ranges by its dependent trips (plan, block id, page): 8192
// tokens of 8/128 bf16 12.1 us (67 MB, 5.5 TB/s), 24 ragged ranges of e4m3 caches with 64-wide heads (27 MB) 7.2, of which 5.2 for the bytes.
// Stores count by requests: with V in pieces of 8 bytes and the lanes of a quad in four rows 13.9 and 8.2, in pieces of 16 12.8 and 7.3, K's lanes four
// to a row 12.3 and 7.1.  Four heads a wave, all asked for at once, took 1 us more.
template <int D, int DT, bool IS_V>
__device__ __forceinline__ void gather_page(const uint8_t *tile, float scale, uint8_t *out, size_t stride, int s0, int s1) {
    // K: token t, a quad's four lanes side by side.  V: element 4 c + r of tokens 4 G .. 4 G + 3, then elements 4 c .. + 3 of token 4 G + r.
    const int lane = threadIdx.x & 63, c = lane & 3, G = lane >> 2 & 3, r = lane >> 4, t = IS_V ? 4 * G + r : lane >> 2;
    constexpr int N = DT == PKV_BF16 ? D / 32 : D / 64;
    u32x4 u[N];
    const u32x4 *unit = reinterpret_cast<const u32x4 *>(tile + (IS_V ? (G * 16 + 4 * c + r) * 16 : (c * 16 + t) * 16));
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = unit[64 * i];
    const bool mine = t >= s0 && t < s1;
    uint8_t *row = out + (ptrdiff_t)(t - s0) * (ptrdiff_t)stride;
    auto values = [&](uint32_t codes) __attribute__((always_inline)) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
        return mk2(pack_bf16_rne(a[0] * scale, a[1] * scale), pack_bf16_rne(b[0] * scale, b[1] * scale));
    };
    auto put8 = [&](int at, u32x4 w) __attribute__((always_inline)) { if (mine) *reinterpret_cast<u32x4 *>(row + 2 * at) = w; };
    // four tokens of element r of a group as 16-bit values -> four elements of token r, between the four rows of 16 lanes
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    auto turned = [&](u32x2 w) __attribute__((always_inline)) {
        const u2 a = __builtin_amdgcn_permlane32_swap(w.x, w.y, false, false);         // now two tokens of elements r & 1 and 2 + (r & 1)
        const u2 b = __builtin_amdgcn_permlane16_swap(__builtin_amdgcn_perm(a.y, a.x, 0x05040100u), __builtin_amdgcn_perm(a.y, a.x, 0x07060302u), false, false);
        return mk2(__builtin_amdgcn_perm(b.y, b.x, 0x05040100u), __builtin_amdgcn_perm(b.y, b.x, 0x07060302u));
    };
    // elements at + 4 c .. + 3 (lo) and at + 16 + 4 c .. + 3 (hi): neighbours exchange, so that either has eight in a row
    auto put_pair = [&](int at, u32x2 lo, u32x2 hi) __attribute__((always_inline)) {
        const bool odd = c & 1;
        auto other = [&](uint32_t x) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false); };
        const uint32_t x = other(odd ? lo.x : hi.x), y = other(odd ? lo.y : hi.y);
        put8(at + 16 * (c & 1) + 8 * (c >> 1), odd ? mk4(x, y, hi.x, hi.y) : mk4(lo.x, lo.y, x, y));
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (DT == PKV_BF16 && !IS_V) {
            put8(8 * (4 * i + c), u[i]);
        } else if constexpr (DT == PKV_BF16) {
            put_pair(32 * i, turned(mk2(u[i].x, u[i].y)), turned(mk2(u[i].z, u[i].w)));
        } else if constexpr (!IS_V) {
            const u32x2 a = values(u[i].x), b = values(u[i].y), g = values(u[i].z), h = values(u[i].w);
            put8(8 * (8 * i + c), mk4(a.x, a.y, b.x, b.y));
            put8(8 * (8 * i + 4 + c), mk4(g.x, g.y, h.x, h.y));
        } else {
#pragma unroll
            for (int k = 0; k < 4; k += 2) put_pair(64 * i + 16 * k, turned(values(u[i][k])), turned(values(u[i][k + 1])));
        }
    }
}

template <int DT>
__global__ __launch_bounds__(64 * PAGE_WAVES) void k_kv_gather(const AttnDesc d, const GatherPlan plan, uint8_t *k_out, uint8_t *v_out) {
    constexpr int E = DT == PKV_BF16 ? 2 : 1;
    const PlanLanes<PKV_PLAN_FEW> lanes(plan.rows);
    // the ranges' sequences and first tokens come with the plan, not behind it
    uint32_t seqs[2], begins[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = (int)(threadIdx.x & 63) + 64 * k, at = i < PKV_PLAN_FEW ? i : PKV_PLAN_FEW - 1;
        seqs[k] = (uint32_t)plan.at[at].seq;
        begins[k] = (uint32_t)plan.at[at].begin;
    }
    asked_for();
    const int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * PAGE_WAVES + (threadIdx.x >> 6)));
    const int which = x & 1, hp = x >> 1, unit = hp / d.Hkv, h = hp - unit * d.Hkv;
    if ((uint32_t)unit >= lanes.units(plan.rows)) return;            // the last work-group may have waves to spare
    const PlanUnit pu = lanes.find(plan.rows, (uint32_t)unit);       // (pu.seq: its place in the list)
    const int place = pu.seq - plan.rows.seq0, seq = (int)lanes.pick(seqs, place), begin = (int)lanes.pick(begins, place), end = begin + pu.rows;
    const int page = begin / PKV_T + pu.unit;
    const int lo = begin > page * PKV_T ? begin : page * PKV_T, hi = end < (page + 1) * PKV_T ? end : (page + 1) * PKV_T;
    const uint32_t id = (uint32_t)PKV_CONST(int32_t, d.table)[(size_t)seq * d.row_stride + page];
    if (id >= d.max_block_id) {
        if ((threadIdx.x & 63) == 0) atomicOr(d.err, 1u);
        return;
    }
    const uint8_t *blk = block_ptr(d, id);
    const float scale = DT == PKV_E4M3 ? reinterpret_cast<const float *>(blk)[(which ? d.Hkv : 0) + h] : 1.f;
    const uint8_t *tile = blk + (DT == PKV_E4M3 ? PKV_FP8_HEADER : 0) + ((size_t)h * 2 + which) * PKV_T * d.D * E;
    const size_t stride = (size_t)d.Hkv * d.D * 2;
    uint8_t *out = (which ? v_out : k_out) + (size_t)(pu.row + lo - begin) * stride + (size_t)h * d.D * 2;
    if (d.D == 128) {
        if (which) gather_page<128, DT, true>(tile, scale, out, stride, lo % PKV_T, lo % PKV_T + hi - lo);
        else gather_page<128, DT, false>(tile, scale, out, stride, lo % PKV_T, lo % PKV_T + hi - lo);
    } else {
        if (which) gather_page<64, DT, true>(tile, scale, out, stride, lo % PKV_T, lo % PKV_T + hi - lo);
        else gather_page<64, DT, false>(tile, scale, out, stride, lo % PKV_T, lo % PKV_T + hi - lo);
    }
}

}  // namespace

hipError_t pkv_launch_kv_gather(const AttnDesc &d, const GatherPlan &plan, void *k_out, void *v_out, hipStream_t s) {
    const unsigned waves = plan.rows.s[plan.rows.n_seqs].unit * (unsigned)d.Hkv * 2u, blocks = (waves + PAGE_WAVES - 1) / PAGE_WAVES;
    if (blocks == 0) return hipSuccess;
    if (d.dtype == PKV_BF16) hipLaunchKernelGGL(k_kv_gather<PKV_BF16>, dim3(blocks), dim3(64 * PAGE_WAVES), 0, s, d, plan, (uint8_t *)k_out, (uint8_t *)v_out);
    else hipLaunchKernelGGL(k_kv_gather<PKV_E4M3>, dim3(blocks), dim3(64 * PAGE_WAVES), 0, s, d, plan, (uint8_t *)k_out, (uint8_t *)v_out);
    return hipGetLastError();
}

hipError_t pkv_launch_kv_write(const AttnDesc &d, int seq, int tok_begin, int n_tok, const void *k, const void *v,
                               const float *ks, const float *vs, int page_tokens, hipStream_t s) {
    (void)page_tokens;
    if (n_tok == 0) return hipSuccess;
    const int32_t *row = d.table + (size_t)seq * d.row_stride;
    const int pages = (tok_begin + n_tok - 1) / PKV_T - tok_begin / PKV_T + 1;
    const unsigned waves = (unsigned)pages * (unsigned)d.Hkv * 2u, blocks = (waves + PAGE_WAVES - 1) / PAGE_WAVES;
    if (d.dtype == PKV_BF16)
        hipLaunchKernelGGL(k_kv_write<PKV_BF16>, dim3(blocks), dim3(64 * PAGE_WAVES), 0, s, d, row, tok_begin, n_tok,
                           (const uint8_t *)k, (const uint8_t *)v, ks, vs);
    else
        hipLaunchKernelGGL(k_kv_write<PKV_E4M3>, dim3(blocks), dim3(64 * PAGE_WAVES), 0, s, d, row, tok_begin, n_tok,
                           (const uint8_t *)k, (const uint8_t *)v, ks, vs);
    return hipGetLastError();
}

hipError_t pkv_launch_kv_read(const AttnDesc &d, int seq, int tok_begin, int n_tok, void *k, void *v, float *ks, float *vs,
                              hipStream_t s) {
    const int64_t total = (int64_t)n_tok * d.Hkv * d.D;
    if (total == 0) return hipSuccess;
    const int32_t *row = d.table + (size_t)seq * d.row_stride;
    const unsigned blocks = (unsigned)((total + 255) / 256);
    if (d.dtype == PKV_BF16)
        hipLaunchKernelGGL(k_kv_read<PKV_BF16>, dim3(blocks), dim3(256), 0, s, d, row, tok_begin, n_tok, (uint8_t *)k,
                           (uint8_t *)v, ks, vs);
    else
        hipLaunchKernelGGL(k_kv_read<PKV_E4M3>, dim3(blocks), dim3(256), 0, s, d, row, tok_begin, n_tok, (uint8_t *)k,
                           (uint8_t *)v, ks, vs);
    return hipGetLastError();
}

hipError_t pkv_launch_kv_append(const AttnDesc &d, const void *k_new, const void *v_new, hipStream_t s) {
    if (d.batch == 0) return hipSuccess;
    const unsigned blocks = (unsigned)(d.batch * d.Hkv);
    if (d.dtype == PKV_BF16)
        hipLaunchKernelGGL(k_kv_append<PKV_BF16>, dim3(blocks), dim3(64), 0, s, d, (const uint16_t *)k_new,
                           (const uint16_t *)v_new);
    else
        hipLaunchKernelGGL(k_kv_append<PKV_E4M3>, dim3(blocks), dim3(64), 0, s, d, (const uint16_t *)k_new,
                           (const uint16_t *)v_new);
    return hipGetLastError();
}

hipError_t pkv_launch_kv_append_chunk(const AttnDesc &d, const ChunkPlan &plan, const void *k_new, const void *v_new, hipStream_t s) {
    const unsigned waves = plan.s[plan.n_seqs].unit * (unsigned)d.Hkv * 2u, blocks = (waves + PAGE_WAVES - 1) / PAGE_WAVES;
    if (blocks == 0) return hipSuccess;
    const dim3 grid(blocks), wg(64 * PAGE_WAVES);
    const uint16_t *k = (const uint16_t *)k_new, *v = (const uint16_t *)v_new;
    if (plan.n_seqs <= PKV_PLAN_FEW) {
        if (d.dtype == PKV_BF16) hipLaunchKernelGGL((k_kv_append_chunk<PKV_BF16, PKV_PLAN_FEW>), grid, wg, 0, s, d, few_of(plan), k, v);
        else hipLaunchKernelGGL((k_kv_append_chunk<PKV_E4M3, PKV_PLAN_FEW>), grid, wg, 0, s, d, few_of(plan), k, v);
    } else {
        if (d.dtype == PKV_BF16) hipLaunchKernelGGL((k_kv_append_chunk<PKV_BF16, PKV_PLAN_SEQS>), grid, wg, 0, s, d, plan, k, v);
        else hipLaunchKernelGGL((k_kv_append_chunk<PKV_E4M3, PKV_PLAN_SEQS>), grid, wg, 0, s, d, plan, k, v);
    }
    return hipGetLastError();
}
