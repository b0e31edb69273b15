"""The operators between a layer's projections and its attention, as cases that can be timed and compared.

Four operators of a serving engine's layer on the shared pool, each in its plain form (elementary torch operations in
32 bits) and, with `own` set, through the calls of `PrismKV`:

  append           `qkv_append[_chunk]`: queries and keys normed head by head, rotated to their positions, and keys and values
                   written into the paged cache, in the cache's type; out of the projection's fused rows.  On an e4m3 cache the
                   values are then read back with `kv_gather`, as an engine does that hands a prompt to another GPU.
  gather           `kv_gather`: cached tokens of several sequences as bf16 rows (swap-out, hand-over, forking a prefix's last tokens)
  decode_prefix    `decode_attention_prefix`: a decode step of sequences that share long prefixes, which are read once for all
  prefill_prefix   `prefill_attention_prefix`: fresh prompts behind a shared prefix

A model is written "q_heads/kv_heads/head_dim dtype".  Lengths are lognormal around a median with sigma `spread` (0: all
equal), at most `cap`; they belong to the case, the seed only deals them to the sequences.  Values are N(0, 1) in bf16;
e4m3 caches hold them quantised per (block, kv head).
"""
import math
import random
import weakref

import numpy as np
import torch

own = False

T = 16                      # tokens per block
DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
EPS = 1e-6

LISTED = [
    # the smallest call: one new token each for four chats of a small model, no norms
    dict(name="append_few", kind="append", model="8/2/64 bf16", batch=4, cached=128, cached_spread=0.8, new=0, new_spread=0.0, cap=256,
         rot=64, layout="half", norm=False, stretch=1.0, before=0),
    # a decode step of a full batch: norms, all of the head rotated, positions behind a shared prefix, stretched for long contexts
    dict(name="append_step", kind="append", model="32/8/128 bf16", batch=64, cached=512, cached_spread=0.8, new=0, new_spread=0.0, cap=2048,
         rot=128, layout="half", norm=True, stretch=8.0, before=4096),
    # a prefill step's chunks, ragged, with neighbouring elements as pairs
    dict(name="append_prompts", kind="append", model="32/8/128 bf16", batch=8, cached=0, cached_spread=0.0, new=512, new_spread=0.5, cap=2048,
         rot=128, layout="pairs", norm=True, stretch=1.0, before=0),
    # prompts that go into an e4m3 cache and from there to another GPU; half of the head rotated
    dict(name="append_hand_over", kind="append", model="32/8/128 e4m3", batch=6, cached=0, cached_spread=0.0, new=400, new_spread=0.6, cap=2048,
         rot=64, layout="half", norm=True, stretch=1.0, before=0),
    # a long sequence is swapped out
    dict(name="gather_swap_out", kind="gather", model="32/8/128 bf16", batch=1, ctx=8192, spread=0.0, cap=8192, skip=0),
    # what prompts hold behind their first tokens, from an e4m3 cache with 64-wide heads, ragged and from inside a block on
    dict(name="gather_tails", kind="gather", model="32/8/64 e4m3", batch=24, ctx=300, spread=0.8, cap=2048, skip=5),
    # few short chats behind a system prompt: latency
    dict(name="decode_prefix_few", kind="decode_prefix", model="8/2/64 bf16", batch=6, groups=1, prefix=320, prefix_spread=0.0, ctx=60,
         spread=0.8, cap=256, alone=1),
    # a full batch behind one system prompt
    dict(name="decode_prefix_batch", kind="decode_prefix", model="32/8/128 bf16", batch=64, groups=1, prefix=4096, prefix_spread=0.0, ctx=400,
         spread=0.8, cap=4096, alone=0),
    # many questions to one long document, the largest decode
    dict(name="decode_prefix_document", kind="decode_prefix", model="64/8/128 bf16", batch=96, groups=1, prefix=24576, prefix_spread=0.0, ctx=256,
         spread=0.5, cap=4096, alone=0),
    # several tenants with prompts of their own on an e4m3 cache, and some requests without
    dict(name="decode_prefix_tenants", kind="decode_prefix", model="32/8/128 e4m3", batch=96, groups=7, prefix=1500, prefix_spread=0.5, ctx=700,
         spread=0.8, cap=4096, alone=9),
    # fresh prompts behind one system prompt
    dict(name="prefill_prefix_prompts", kind="prefill_prefix", model="32/8/128 bf16", batch=16, groups=1, prefix=2048, prefix_spread=0.0, cached=0,
         new=160, spread=0.6, cap=1024, alone=0),
    # the same on an e4m3 cache with 64-wide heads and several prefixes; some prompts have a part of their own cached
    dict(name="prefill_prefix_tenants", kind="prefill_prefix", model="32/8/64 e4m3", batch=20, groups=4, prefix=700, prefix_spread=0.5, cached=64,
         new=90, spread=0.7, cap=1024, alone=3),
]


def listed():
    return [dict(c) for c in LISTED]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = [max(work(c)[w] for c in LISTED) for w in ("bytes", "flops")]
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            return case


def _draw(rng):
    kind = rng.choice(["append", "append", "gather", "decode_prefix", "decode_prefix", "decode_prefix", "prefill_prefix", "prefill_prefix"])
    hkv, d = rng.choice([1, 2, 4, 5, 8, 8]), rng.choice([64, 128, 128])
    model = "%d/%d/%d %s" % (hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), hkv, d, rng.choice(["bf16", "bf16", "e4m3"]))
    spread = rng.choice([0.0, 0.5, 0.8])
    if kind == "append":
        e4m3 = model.endswith("e4m3")
        new = rng.choice([0, 0, _logint(rng, 2, 1500), _logint(rng, 17, 1500)]) if not e4m3 else _logint(rng, 2, 1500)
        batch = _logint(rng, 1, max(1, min(128, 6000 // max(new, 1))))
        cached = 0 if e4m3 else rng.choice([0, _logint(rng, 1, 600)])
        return dict(kind=kind, model=model, batch=batch, cached=cached, cached_spread=spread, new=new, new_spread=rng.choice([0.0, 0.7]), cap=2048,
                    rot=rng.choice([d, d, d // 2, d // 4, 16, 3 * d // 4]), layout=rng.choice(["half", "half", "pairs"]), norm=rng.random() < 0.6,
                    stretch=rng.choice([1.0, 1.0, 4.0, 32.0]), before=rng.choice([0, 16 * _logint(rng, 1, 6000)]))
    if kind == "gather":
        ctx = _logint(rng, 3, 8000)
        return dict(kind=kind, model=model, batch=_logint(rng, 1, max(1, min(64, 9000 // ctx))), ctx=ctx, spread=spread, cap=8192,
                    skip=rng.choice([0, 0, rng.randint(1, 40)]))
    batch = _logint(rng, 2, 128) if kind == "decode_prefix" else _logint(rng, 1, 32)
    groups = rng.choice([1, 1, rng.randint(1, max(1, batch // 3))])
    prefix = _logint(rng, 16, max(20, min(24000, 60000 // groups)))
    alone = rng.choice([0, 0, rng.randint(0, batch // 3)])
    case = dict(kind=kind, model=model, batch=batch, groups=groups, prefix=prefix, prefix_spread=rng.choice([0.0, 0.6]))
    if kind == "decode_prefix":
        case |= dict(ctx=_logint(rng, 1, max(2, min(3000, 100000 // batch))), spread=spread, cap=4096, alone=alone)
    else:
        case |= dict(cached=rng.choice([0, 0, _logint(rng, 4, 500)]), new=_logint(rng, 1, max(2, min(700, 4000 // batch))), spread=spread, cap=1024, alone=alone)
    return case


# ---------------------------------------------------------------- what a case says

class Spec:
    def __init__(self, text):
        heads, dtype = text.split()
        self.hq, self.hkv, self.d = (int(x) for x in heads.split("/"))
        self.g = self.hq // self.hkv
        self.e4m3 = dtype == "e4m3"

    def kv_bytes(self, tokens, blocks):
        """K and V of so many cached tokens, and the scales of so many blocks."""
        return tokens * self.hkv * self.d * 2 * (1 if self.e4m3 else 2) + (blocks * self.hkv * 8 if self.e4m3 else 0)


def _blocks(tokens):
    return (tokens + T - 1) // T


def _rng(case, what):
    return random.Random("%s %s" % (what, sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(rng, n, median, spread, cap, least=1):
    return [min(cap, max(least, int(round(median * math.exp(spread * rng.gauss(0.0, 1.0)))))) for _ in range(n)]


def _deal(seed, values):
    values = list(values)
    random.Random("deal %d" % seed).shuffle(values)
    return values


def _layout(case):
    """Lengths of a case, before the seed deals them to the sequences.  append: (cached, new tokens) of each sequence, one new one in a
    decode step; gather: tokens held; otherwise blocks of each prefix and (group or -1, own tokens before, new tokens)."""
    rng, n = _rng(case, "layout"), case["batch"]
    if case["kind"] == "append":
        old = _lengths(rng, n, case["cached"], case["cached_spread"], case["cap"], 0) if case["cached"] else [0] * n
        return list(zip(old, _lengths(rng, n, case["new"], case["new_spread"], case["cap"]) if case["new"] else [1] * n))
    if case["kind"] == "gather":
        return [x + case["skip"] for x in _lengths(rng, n, case["ctx"], case["spread"], case["cap"])]
    blocks = [max(1, x // T) for x in _lengths(rng, case["groups"], case["prefix"], case["prefix_spread"], 2 * case["prefix"], T)]
    # every group has a member, the others go where they may
    group = [-1] * case["alone"] + list(range(case["groups"]))
    group = (group + [rng.randrange(case["groups"]) for _ in range(n)])[:n]
    if case["kind"] == "decode_prefix":
        own_tokens = [(0, x) for x in _lengths(rng, n, case["ctx"], case["spread"], case["cap"])]
    else:
        old = _lengths(rng, n, case["cached"], 0.8, case["cap"], 0) if case["cached"] else [0] * n
        own_tokens = list(zip(old, _lengths(rng, n, case["new"], case["spread"], case["cap"])))
    return blocks, [(g, o, w) for g, (o, w) in zip(group, own_tokens)]


def work(case):
    s, kind = Spec(case["model"]), case["kind"]
    if kind == "append":
        new = sum(w for _, w in _layout(case))
        blocks = sum(_blocks(w) for _, w in _layout(case))
        nbytes = new * (s.hq + 2 * s.hkv) * s.d * 2 + new * s.hq * s.d * 2 + s.kv_bytes(new, blocks) + new * s.hkv * s.d * 4 * s.e4m3 + s.kv_bytes(new, blocks) * s.e4m3
        return {"bytes": nbytes, "flops": 10 * new * (s.hq + s.hkv) * s.d}
    if kind == "gather":
        ctx = [x - case["skip"] for x in _layout(case)]
        return {"bytes": s.kv_bytes(sum(ctx), sum(_blocks(x) for x in ctx)) + sum(ctx) * s.hkv * s.d * 4, "flops": 0}
    blocks, seqs = _layout(case)
    held = [o + w for _, o, w in seqs]
    nbytes = s.kv_bytes(sum(blocks) * T + sum(held), sum(blocks) + sum(_blocks(x) for x in held))
    seen = rows = 0
    for g, o, w in seqs:
        p = T * blocks[g] if g >= 0 else 0
        if kind == "decode_prefix":
            rows, seen = rows + 1, seen + p + w
        else:
            rows, seen = rows + w, seen + w * (p + o) + w * (w + 1) // 2
    return {"bytes": nbytes + rows * s.hq * s.d * 6, "flops": 4 * s.d * s.hq * seen}


# ---------------------------------------------------------------- inputs

def _gen(seed, *key):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + sum((k + 1) * 7919 ** (i + 1) for i, k in enumerate(key))) % (1 << 62))
    return g


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _cache(s, lens, g):
    """K and V of sequences of so many tokens, padded to the longest: [n][blocks][T][Hkv][D] bf16, or e4m3 with scales [n][blocks][Hkv]."""
    kv = []
    for _ in range(2):
        x = _randn((len(lens), max(1, max(_blocks(n) for n in lens)), T, s.hkv, s.d), g)
        scale = None
        if s.e4m3:
            y = x.float()
            scale = y.abs().amax(dim=(2, 4)) / E4M3_MAX
            x = (y / scale[:, :, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(E4M3)
        kv.append((x, scale))
    return kv


def _frequencies(case):
    """Radians a token of the pairs, 64 bits: base 10000; stretched (for contexts `stretch` times those of training, 4096 tokens) where a pair
    turns less than once over a trained context, not where it turns more than four times, and in between in proportion."""
    n = case["rot"] // 2
    f = 10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)
    if case["stretch"] != 1.0:
        keep = ((4096.0 * f / (2 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * keep + f / case["stretch"] * (1.0 - keep)
    return f


def _magnitude(case):
    return 0.1 * math.log(case["stretch"]) + 1.0


class State:
    pass


def _close(be, pool, model, rows, rotary):
    torch.cuda.synchronize()
    if rotary is not None:
        be.rotary_destroy(rotary)
    be.seq_release_batch(model, np.arange(rows, dtype=np.int32))
    be.balloon_resize(model, 0)
    be.model_unregister(model)
    be.pool_destroy(pool)
    torch.cuda.synchronize()


def _open(st, s, lens, one_block_frames=False, seed=0):
    """A pool with one model whose rows 0, 1, ... have room for so many tokens.  With frames of one block handed out in order, row by
    row, the rows' blocks lie side by side in the pool; otherwise rows grow side by side on scattered frames."""
    from paper_2505_04021_amd import PKV_BF16, PKV_E4M3, PrismKV
    be = st.be = PrismKV(DEV)
    block = 2 * T * s.hkv * s.d * (1 if s.e4m3 else 2) + (128 if s.e4m3 else 0)
    blocks = [max(1, _blocks(n)) for n in lens]
    st.max_blocks = max(blocks)
    if one_block_frames:
        frame, need = block, len(lens) * st.max_blocks
        st.storage = torch.zeros(need * frame, dtype=torch.uint8, device=DEV)
        st.pool = be.pool_create(need * frame, T, frame, st.storage)
    else:
        frame = 2 << 20
        need = (sum(blocks) + frame // block - 1) // (frame // block)
        n_frames = 2 * need + 64
        st.pool = be.pool_create(n_frames * frame, T, frame)
        order = list(range(n_frames))
        random.Random("frames %d" % seed).shuffle(order)
        assert be.pool_seed_free_order(st.pool, np.array(order, dtype=np.uint32)) == 0
    assert st.pool >= 0, be.last_error()
    m = st.m = be.model_register(st.pool, s.hq, s.hkv, s.d, PKV_E4M3 if s.e4m3 else PKV_BF16, len(lens), st.max_blocks)
    assert m >= 0 and be.balloon_resize(m, need) == need
    rows = np.arange(len(lens), dtype=np.int32)
    if one_block_frames:
        be.seq_reserve_batch(m, rows, np.full(len(lens), st.max_blocks * T, dtype=np.int32))
    else:
        for upto in range(256, st.max_blocks * T + 256, 256):
            some = [i for i in rows if min(lens[i], upto) > upto - 256]
            for a in range(0, len(some), 4096):
                assert be.seq_reserve_batch(m, some[a:a + 4096], [min(lens[i], upto) for i in some[a:a + 4096]]) >= 0
    weakref.finalize(st, _close, be, st.pool, m, len(lens), getattr(st, "rotary", None))


def _fill(st, s, row, n, cache, i):
    """The first n tokens of cache entry i into row `row`."""
    if n == 0:
        return
    (k, ks), (v, vs) = cache
    b = _blocks(n)
    rows = [x[i, :b].reshape(b * T, s.hkv, s.d)[:n].contiguous().view(torch.uint8 if s.e4m3 else torch.int16) for x in (k, v)]
    assert st.be.kv_write(st.m, row, 0, rows[0], rows[1], ks[i, :b] if s.e4m3 else None, vs[i, :b] if s.e4m3 else None) == n


def prepare(case, seed):
    s, kind, g = Spec(case["model"]), case["kind"], _gen(seed)
    st = State()
    st.case, st.s = case, s
    if kind == "append":
        seqs = _deal(seed, _layout(case))
        st.new, st.ctx_host = [w for _, w in seqs], [o + w for o, w in seqs]
        st.ctx, st.q_lens = _i32(st.ctx_host), np.array(st.new, dtype=np.int32)
        st.before = _i32([case["before"] + 3 * i for i in range(case["batch"])])
        rows = sum(st.new)
        fused = _randn((rows, s.hq + 2 * s.hkv, s.d), g)
        st.q, st.k, st.v = fused[:, :s.hq], fused[:, s.hq:s.hq + s.hkv], fused[:, s.hq + s.hkv:]
        st.qw, st.kw = ((1.0 + 0.2 * _randn((s.d,), g).float()).to(torch.bfloat16) for _ in range(2)) if case["norm"] else (None, None)
        st.freq, st.magnitude = _frequencies(case), _magnitude(case)
        if own:
            from paper_2505_04021_amd import PrismKV, ROTARY_HALF, ROTARY_PAIRS
            st.rotary = PrismKV(DEV).rotary_create(case["rot"], ROTARY_HALF if case["layout"] == "half" else ROTARY_PAIRS, st.freq.numpy(), st.magnitude)
            assert st.rotary >= 0
            _open(st, s, st.ctx_host, one_block_frames=not s.e4m3)
            st.q_out = torch.empty((rows, s.hq, s.d), dtype=torch.bfloat16, device=DEV)
            if s.e4m3:
                st.k_back, st.v_back = (torch.empty((rows, s.hkv, s.d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
                st.every, st.zeros = np.arange(case["batch"], dtype=np.int32), np.zeros(case["batch"], dtype=np.int32)
            else:
                # the pool's bytes by sequence, block and token: no copy, a view of the blocks' own order of elements
                x = st.storage.view(torch.bfloat16).view(case["batch"], st.max_blocks, s.hkv, 2, T * s.d)
                st.k_view = x[:, :, :, 0].view(case["batch"], st.max_blocks, s.hkv, s.d // 8, T, 8).permute(0, 1, 4, 2, 3, 5)
                st.v_view = x[:, :, :, 1].view(case["batch"], st.max_blocks, s.hkv, s.d // 32, 4, 16, 2, 4).permute(0, 1, 4, 7, 2, 3, 6, 5)
        else:
            blocks = max(_blocks(x) for x in st.ctx_host)
            seq = torch.repeat_interleave(torch.arange(case["batch"]), torch.tensor(st.new))
            index = torch.cat([torch.arange(o, o + w) for o, w in seqs])
            st.seq, st.index = seq.to(DEV), index.to(DEV)          # each row's sequence and its index in it: the plain form's plan
            if not s.e4m3:
                st.k_cache, st.v_cache = (torch.zeros((case["batch"], blocks * T, s.hkv, s.d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return st
    if kind == "gather":
        lens = st.lens = _deal(seed, _layout(case))
        st.skip = case["skip"]
        st.cache = _cache(s, lens, g)
        rows = sum(lens) - st.skip * len(lens)
        if own:
            _open(st, s, lens, seed=seed)
            for i, n in enumerate(lens):
                _fill(st, s, i, n, st.cache, i)
            st.seqs, st.begin = np.arange(len(lens), dtype=np.int32), np.full(len(lens), st.skip, dtype=np.int32)
            st.count = np.array(lens, dtype=np.int32) - st.skip
            st.k_back, st.v_back = (torch.empty((rows, s.hkv, s.d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            del st.cache
        else:
            blocks = st.cache[0][0].shape[1]
            st.rows = torch.cat([torch.arange(i * blocks * T + st.skip, i * blocks * T + n) for i, n in enumerate(lens)]).to(DEV)
        return st
    st.blocks, seqs = _layout(case)
    seqs = _deal(seed, seqs)
    st.group, st.old, st.new = ([x[i] for x in seqs] for i in range(3))
    held = [o + w for _, o, w in seqs]
    n, groups = len(seqs), len(st.blocks)
    rows = n if kind == "decode_prefix" else sum(st.new)
    st.q = _randn((rows, s.hq, s.d), g)
    st.held = held
    prefix, tail = _cache(s, [b * T for b in st.blocks], g), _cache(s, held, g)
    if own:
        _open(st, s, held + [b * T for b in st.blocks], seed=seed)     # the prefixes' rows behind the sequences'
        for i, x in enumerate(held):
            _fill(st, s, i, x, tail, i)
        for j, b in enumerate(st.blocks):
            _fill(st, s, n + j, b * T, prefix, j)
        st.ctx, st.q_lens = _i32(held), np.array(st.new, dtype=np.int32)
        st.prefix_seqs = np.array([n + x if x >= 0 else -1 for x in st.group], dtype=np.int32)
        st.prefix_blocks = np.array([st.blocks[x] if x >= 0 else 0 for x in st.group], dtype=np.int32)
        st.out = torch.empty(st.q.shape, dtype=torch.float32, device=DEV)
    else:
        st.prefix, st.tail = prefix, tail
        members = [[i for i in range(n) if st.group[i] == j] for j in range(groups)]
        most = max(1, max(len(x) for x in members))
        st.members = torch.tensor([x + [0] * (most - len(x)) for x in members], device=DEV)
        at = [members[x].index(i) if x >= 0 else 0 for i, x in enumerate(st.group)]
        st.place = torch.tensor([max(x, 0) * most + a for x, a in zip(st.group, at)], device=DEV)
        st.has, st.lens, st.prefix_lens = (torch.tensor(x, device=DEV) for x in ([x >= 0 for x in st.group], held, [b * T for b in st.blocks]))
        if kind == "prefill_prefix":
            longest = max(st.new)
            row0 = np.cumsum([0] + st.new)
            st.rows = torch.tensor([[row0[i] + min(j, st.new[i] - 1) for j in range(longest)] for i in range(n)], device=DEV)
            st.back = torch.cat([torch.arange(w) + i * longest for i, w in enumerate(st.new)]).to(DEV)
            st.first = torch.tensor(st.old, device=DEV)
    return st


# ---------------------------------------------------------------- one pass

def _values(cache):
    """Cached values in 32 bits, [n][tokens][Hkv][D]."""
    x, scale = cache
    y = x.float()
    if scale is not None:
        y = y * scale[:, :, None, :, None]
    return y.flatten(1, 2)


def _turned(x, weight, st):
    """x [rows][heads][D] normed, if there is a weight, and rotated: 32 bits, angles in 64."""
    c = st.case
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + EPS) * weight.float()
    angle = (st.before.double()[st.seq] + st.index.double())[:, None] * st.freq.to(DEV)
    cos, sin = ((f(angle) * st.magnitude).float()[:, None, :] for f in (torch.cos, torch.sin))
    r = c["rot"]
    if c["layout"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., r:]], dim=-1).to(torch.bfloat16)
    a, b = y[..., 0:r:2], y[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2), y[..., r:]], dim=-1).to(torch.bfloat16)


def _requantised(x, st):
    """What an e4m3 cache gives back of rows x [rows][Hkv][D] appended to sequences from token 0 on: one scale for a block and kv head, the
    largest amax / 448 so far; where a token raises it, the codes before are encoded again."""
    s, n = st.s, len(st.new)
    blocks = max(_blocks(w) for w in st.new)
    y = torch.zeros((n, blocks * T, s.hkv, s.d), device=DEV)
    y[st.seq, st.index] = x.float()
    y = y.view(n * blocks, T, s.hkv, s.d)
    there = torch.zeros((n, blocks * T), dtype=torch.bool, device=DEV)
    there[st.seq, st.index] = True
    there = there.view(n * blocks, T)
    encode = lambda v: v.clamp(-E4M3_MAX, E4M3_MAX).to(E4M3).float()  # noqa: E731
    cand = y.abs().amax(dim=-1) / torch.full((), E4M3_MAX, device=DEV)          # (a number would be a product with its reciprocal)
    scale = torch.where(cand[:, 0] > 0, cand[:, 0], torch.ones_like(cand[:, 0]))
    codes = torch.zeros_like(y)
    for t in range(T):
        up = torch.where(there[:, t, None], torch.maximum(scale, cand[:, t]), scale)
        codes = torch.where((up > scale)[:, None, :, None], encode(codes * scale[:, None, :, None] / up[:, None, :, None]), codes)
        scale = up
        codes[:, t] = torch.where(there[:, t, None, None], encode(y[:, t] / scale[:, :, None]), codes[:, t])
    back = (codes * scale[:, None, :, None]).view(n, blocks * T, s.hkv, s.d)
    return back[st.seq, st.index].to(torch.bfloat16)


def _softmax_sums(scores, seen, v):
    """Unnormalised: maxima, sums and products with v of scores [..., rows, tokens]; a row that sees nothing has maximum -inf and sums of zero."""
    scores = scores.masked_fill(~seen, -math.inf)
    m = scores.amax(dim=-1, keepdim=True)
    p = torch.exp(scores - m.clamp_min(torch.finfo(torch.float32).min))
    return m, p.sum(dim=-1, keepdim=True), torch.matmul(p, v)


def _joined(a, b):
    m = torch.maximum(a[0], b[0]).clamp_min(torch.finfo(torch.float32).min)
    fa, fb = torch.exp(a[0] - m), torch.exp(b[0] - m)
    den = fa * a[1] + fb * b[1]
    return torch.where(den > 0, (fa * a[2] + fb * b[2]) / den, torch.zeros_like(den))


def _plain_attention(st):
    s, n, prefill = st.s, len(st.new), st.case["kind"] == "prefill_prefix"
    q = (st.q[st.rows] if prefill else st.q[:, None]).float() / math.sqrt(s.d)        # [n][tokens][Hq][D], a ragged chunk's last token repeated
    tokens = q.shape[1]
    q = q.view(n, tokens, s.hkv, s.g, s.d).permute(0, 2, 1, 3, 4).reshape(n, s.hkv, tokens * s.g, s.d)
    # the prefixes: columns of all members side by side
    k, v = (_values(x).permute(0, 2, 1, 3).contiguous() for x in st.prefix)
    groups, most = st.members.shape
    cols = q[st.members].permute(0, 2, 1, 3, 4).reshape(groups, s.hkv, most * tokens * s.g, s.d)
    seen = (torch.arange(k.shape[2], device=DEV)[None] < st.prefix_lens[:, None])[:, None, None]
    a = _softmax_sums(torch.matmul(cols, k.transpose(-1, -2)), seen, v)
    a = [x.view(groups, s.hkv, most, tokens * s.g, -1).permute(0, 2, 1, 3, 4).flatten(0, 1)[st.place] for x in a]
    a[0] = a[0].masked_fill(~st.has[:, None, None, None], -math.inf)
    # their own tokens
    k, v = (_values(x).permute(0, 2, 1, 3).contiguous() for x in st.tail)
    at = torch.arange(k.shape[2], device=DEV)
    if prefill:
        last = st.first[:, None] + torch.arange(tokens, device=DEV)[None]
        seen = (at <= last[..., None]).repeat_interleave(s.g, dim=1)[:, None]
    else:
        seen = (at < st.lens[:, None])[:, None, None]
    b = _softmax_sums(torch.matmul(q, k.transpose(-1, -2)), seen, v)
    out = _joined(a, b).view(n, s.hkv, tokens, s.g, s.d).permute(0, 2, 1, 3, 4).reshape(n * tokens, s.hq, s.d)
    return out[st.back] if prefill else out


def run(st):
    kind, s = st.case["kind"], st.s
    if own:
        be, m = st.be, st.m
        if kind == "append":
            if st.case["new"]:
                be.qkv_append_chunk_dev(m, st.q, st.k, st.v, st.q_lens, st.ctx, st.q_out, st.qw, st.kw, EPS, st.rotary, st.before)
            else:
                be.qkv_append_dev(m, st.q, st.k, st.v, st.ctx, st.q_out, st.qw, st.kw, EPS, st.rotary, st.before)
            if s.e4m3:
                be.kv_gather_dev(m, st.every, st.zeros, st.q_lens, st.k_back, st.v_back)
                return st.q_out, st.k_back, st.v_back
            return st.q_out, st.k_view, st.v_view
        if kind == "gather":
            be.kv_gather_dev(m, st.seqs, st.begin, st.count, st.k_back, st.v_back)
            return st.k_back, st.v_back
        if kind == "decode_prefix":
            be.decode_attention_prefix_dev(m, st.q, st.prefix_seqs, st.prefix_blocks, st.ctx, st.out)
        else:
            be.prefill_attention_prefix_dev(m, st.q, st.q_lens, st.prefix_seqs, st.prefix_blocks, st.ctx, st.out)
        return st.out
    if kind == "append":
        q, k = _turned(st.q, st.qw, st), _turned(st.k, st.kw, st)
        if s.e4m3:
            return q, _requantised(k, st), _requantised(st.v, st)
        st.k_cache[st.seq, st.index] = k
        st.v_cache[st.seq, st.index] = st.v
        n = len(st.new)
        return q, st.k_cache.view(n, -1, T, s.hkv, s.d // 8, 8), st.v_cache.view(n, -1, 4, 4, s.hkv, s.d // 32, 2, 16)
    if kind == "gather":
        return tuple(_values(x).flatten(0, 1)[st.rows].to(torch.bfloat16) for x in st.cache)
    return _plain_attention(st)


# ---------------------------------------------------------------- the same in 64 bits

def _exact_turn(row, weight, pos, freq, magnitude, case):
    """One token's heads [heads][D] in 64 bits, element pairs as complex numbers."""
    y = row.double()
    if weight is not None:
        y = weight.double() * y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / y.shape[-1] + EPS)
    r, h = case["rot"], case["rot"] // 2
    first, second = (y[..., :, :h], y[..., :, h:r]) if case["layout"] == "half" else (y[..., :, 0:r:2], y[..., :, 1:r:2])
    z = torch.complex(first, second) * torch.polar(torch.full_like(freq, magnitude), freq * pos)
    y = y.clone()
    if case["layout"] == "half":
        y[..., :, :h], y[..., :, h:r] = z.real, z.imag
    else:
        y[..., :, 0:r:2], y[..., :, 1:r:2] = z.real, z.imag
    return y


def _exact_codes(rows):
    """What a block's e4m3 cache holds after the tokens rows [n <= T][Hkv][D] (bf16 values) have come one after the other, as values."""
    rnd = lambda v: v.float().clamp(-E4M3_MAX, E4M3_MAX).to(E4M3).float()  # noqa: E731
    held, scale = None, None
    for x in rows.float():
        cand = x.abs().amax(-1, keepdim=True) / torch.tensor(E4M3_MAX, device=DEV)
        if held is None:
            scale = torch.where(cand > 0, cand, torch.ones_like(cand))
            held = rnd(x / scale)[None]
        else:
            up = torch.maximum(cand, scale)
            held = torch.where(up > scale, rnd(held * scale / up), held)
            scale = up
            held = torch.cat([held, rnd(x / scale)[None]])
    return held.double() * scale.double()


def _exact_rows(q, k, v, limits):
    """softmax(q K^T / sqrt(D)) V in 64 bits: q [n][Hq][D], k and v [tokens][Hkv][D]; row i sees the first limits[i] tokens."""
    n, hq, d = q.shape
    hkv = k.shape[1]
    out = torch.zeros((n, hq, d), dtype=torch.float64, device=DEV)
    if k.shape[0] == 0:
        return out
    late = torch.arange(k.shape[0], device=DEV)[None, :] >= torch.tensor(limits, device=DEV)[:, None]
    for h in range(hkv):
        for j in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
            z = (q[:, j].double() @ k[:, h].t().contiguous()) * d ** -0.5
            out[:, j] = torch.softmax(z.masked_fill(late, -math.inf), dim=-1) @ v[:, h].contiguous()
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    s, kind = st.s, case["kind"]
    dequantised = lambda c, i: (c[0][i].double() * (c[1][i].double()[:, None, :, None] if c[1] is not None else 1.0)).flatten(0, 1)  # noqa: E731
    if kind == "append":
        freq = st.freq.to(DEV)
        pos = (st.before.long()[st.seq] + st.index).double()[:, None, None]
        q, k = _exact_turn(st.q, st.qw, pos, freq, st.magnitude, case), _exact_turn(st.k, st.kw, pos, freq, st.magnitude, case)
        if s.e4m3:
            back, at = [[], []], 0
            for w in st.new:
                for j, x in enumerate((k.to(torch.bfloat16), st.v)):
                    back[j] += [_exact_codes(x[at + b:at + min(b + T, w)]) for b in range(0, w, T)]
                at += w
            return q, torch.cat(back[0]), torch.cat(back[1])
        caches = []
        for x in (k, st.v.double()):
            c = torch.zeros((len(st.new), max(_blocks(n) for n in st.ctx_host) * T, s.hkv, s.d), dtype=torch.float64, device=DEV)
            c.index_put_((st.seq, st.index), x)
            caches.append(c)
        n = len(st.new)
        return q, caches[0].reshape(n, -1, T, s.hkv, s.d // 8, 8), caches[1].reshape(n, -1, 4, 4, s.hkv, s.d // 32, 2, 16)
    if kind == "gather":
        return tuple(torch.cat([dequantised(c, i)[st.skip:n] for i, n in enumerate(st.lens)]) for c in st.cache)
    answers, row = [], 0
    for i, (g, o, w) in enumerate(zip(st.group, st.old, st.new)):
        k, v = ([dequantised(c, i)[:o + w]] for c in st.tail)
        if g >= 0:
            k, v = ([dequantised(c, g)[:T * st.blocks[g]]] + x for c, x in zip(st.prefix, (k, v)))
        k, v = torch.cat(k), torch.cat(v)
        n = 1 if kind == "decode_prefix" else w
        limits = [k.shape[0] - (n - 1) + j for j in range(n)]
        answers.append(_exact_rows(st.q[row:row + n], k, v, limits))
        row += n
    return torch.cat(answers)
