"""Attention with sliding windows and sinks, and drafted trees over the paged cache, as cases that can be timed and compared.

Five operators of a serving engine on the shared pool, each in its plain form (elementary torch operations in 32 bits) and,
with `own` set, through the calls of `PrismKV`:

  window_decode    `decode_attention_window`: a decode step whose queries see the last `window` tokens and the first `sinks`
  window_prefill   `prefill_attention_window`: the same for chunks of new tokens
  tree             `tree_attention`: trees of drafted tokens verified over the cache, each token seeing the context and its ancestors
  draft            `qkv_append_tree` for every layer and `kv_keep`: drafted tokens go into the cache at the positions of their depths,
                   and those of an accepted path are moved together.  What an e4m3 cache then holds is read back with `kv_gather`.

A model is written "q_heads/kv_heads/head_dim dtype".  Lengths are lognormal around a median with sigma `spread` (0: all
equal), at most `cap`; they and the trees belong to the case, the seed only deals them to the sequences.  Values are N(0, 1) in
bf16; e4m3 caches hold them quantised per (block, kv head).
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
BAND = 128                  # queries of a block of the plain banded form

LISTED = [
    # the smallest call: four chats of a small model, some shorter than the window
    dict(name="window_few", kind="window_decode", model="8/2/64 bf16", batch=4, ctx=200, spread=0.8, cap=1024, window=128, sinks=4),
    # a decode step of a full batch whose contexts are several windows long
    dict(name="window_batch", kind="window_decode", model="32/8/128 bf16", batch=64, ctx=6000, spread=0.5, cap=16384, window=1024, sinks=4),
    # the largest decode: a wide window on an e4m3 cache, an odd number of sinks
    dict(name="window_wide", kind="window_decode", model="64/8/128 e4m3", batch=96, ctx=7000, spread=0.3, cap=12288, window=4096, sinks=19),
    # whole prompts, several windows long
    dict(name="window_prompts", kind="window_prefill", model="32/8/128 bf16", batch=6, cached=0, new=1500, spread=0.4, cap=4096, window=512, sinks=4),
    # chunks of long prompts in front of a wide window, no sinks
    dict(name="window_chunks", kind="window_prefill", model="32/8/64 e4m3", batch=5, cached=9000, new=512, spread=0.2, cap=16384, window=2000, sinks=0),
    # a few drafted tokens for four chats of a small model: latency
    dict(name="tree_few", kind="tree", model="8/2/64 bf16", batch=4, cached=250, spread=0.8, cap=1024, nodes=5, branch=0.3, window=0, sinks=0),
    # short drafts of a full batch, hardly branched: 16 columns a kv head
    dict(name="tree_chains", kind="tree", model="32/8/128 bf16", batch=64, cached=1000, spread=0.7, cap=8192, nodes=4, branch=0.1, window=0, sinks=0),
    # branched drafts of a batch
    dict(name="tree_batch", kind="tree", model="32/8/128 bf16", batch=32, cached=1500, spread=0.6, cap=8192, nodes=26, branch=0.5, window=0, sinks=0),
    # large trees behind long documents: most products
    dict(name="tree_long", kind="tree", model="64/8/128 bf16", batch=3, cached=20000, spread=0.2, cap=32768, nodes=60, branch=0.6, window=0, sinks=0),
    # drafts verified by a layer with a window, on an e4m3 cache: 28 columns
    dict(name="tree_window", kind="tree", model="32/8/128 e4m3", batch=48, cached=2500, spread=0.6, cap=8192, nodes=7, branch=0.4, window=1024, sinks=4),
    # drafted tokens of four chats into the cache and the accepted ones together: latency
    dict(name="draft_few", kind="draft", model="8/2/64 bf16", batch=4, cached=50, spread=0.5, cap=128, nodes=5, branch=0.3, layers=1, rot=64, layout="half",
         norm=False),
    # the same for all layers of a small stack and a batch of branched drafts, with norms
    dict(name="draft_layers", kind="draft", model="32/8/128 bf16", batch=32, cached=60, spread=0.5, cap=128, nodes=26, branch=0.5, layers=8, rot=128, layout="half",
         norm=True),
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
    kind = rng.choice(["window_decode", "window_decode", "window_prefill", "window_prefill", "tree", "tree", "tree", "draft"])
    hkv, d = rng.choice([1, 2, 4, 5, 8, 8]), rng.choice([64, 128, 128])
    model = "%d/%d/%d %s" % (hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), hkv, d, rng.choice(["bf16", "bf16", "e4m3"]))
    spread = rng.choice([0.0, 0.5, 0.8])
    sinks = rng.choice([0, 1, 4, 16, rng.randint(2, 100)])
    if kind == "window_decode":
        batch = _logint(rng, 1, 128)
        return dict(kind=kind, model=model, batch=batch, ctx=_logint(rng, 1, max(2, min(12000, 500000 // batch))), spread=spread, cap=12288,
                    window=_logint(rng, 1, 6000), sinks=sinks)
    if kind == "window_prefill":
        new = _logint(rng, 1, 1500)
        batch = _logint(rng, 1, max(1, min(48, 8000 // new)))
        return dict(kind=kind, model=model, batch=batch, cached=rng.choice([0, 0, _logint(rng, 1, max(2, min(9000, 90000 // batch)))]), new=new, spread=spread, cap=12288,
                    window=_logint(rng, 1, 4000), sinks=sinks)
    nodes = _logint(rng, 1, 128)
    batch = _logint(rng, 1, max(1, min(128, 2500 // nodes)))
    case = dict(kind=kind, model=model, batch=batch, spread=spread, nodes=nodes, branch=rng.choice([0.0, 0.2, 0.5, 0.8]))
    if kind == "tree":
        case |= dict(cached=rng.choice([0, _logint(rng, 1, max(2, min(16000, 120000 // batch)))]), cap=16384,
                     window=rng.choice([0, 0, _logint(rng, nodes, 4000)]), sinks=sinks)
    else:
        case |= dict(cached=rng.choice([0, _logint(rng, 1, 100)]), cap=128, layers=rng.choice([1, 1, 2, 5]), rot=rng.choice([d, d, d // 2, 16]),
                     layout=rng.choice(["half", "half", "pairs"]), norm=rng.random() < 0.6)
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


def _tree(rng, n, branch):
    """Parents of n drafted tokens, each before its children (-1: behind the context): a token continues the one before it, or with
    probability `branch` any earlier one or the context."""
    return [i - 1 if rng.random() >= branch else rng.randrange(-1, i) if i else -1 for i in range(n)]


def _path(rng, parents):
    """An accepted path: a token without children and the ancestors of it, cut somewhere behind its first token."""
    at, path = rng.choice([i for i in range(len(parents)) if i not in parents]), []
    while at >= 0:
        path.append(at)
        at = parents[at]
    return path[::-1][:rng.randint(1, len(path))]


def _layout(case):
    """Lengths and trees of a case, before the seed deals them to the sequences: (cached tokens before, new tokens, parents of drafted
    tokens, accepted path)."""
    rng, n = _rng(case, "layout"), case["batch"]
    if case["kind"] == "window_decode":
        return [(x - 1, 1, None, None) for x in _lengths(rng, n, case["ctx"], case["spread"], case["cap"])]
    old = _lengths(rng, n, case["cached"], case["spread"], case["cap"], 0) if case["cached"] else [0] * n
    if case["kind"] == "window_prefill":
        return [(o, w, None, None) for o, w in zip(old, _lengths(rng, n, case["new"], case["spread"], 2 * case["new"]))]
    if case["kind"] == "draft" and case["model"].endswith("e4m3"):
        old = [x // T * T for x in old]          # drafts that begin a block: its scales then start afresh in every pass
    seqs = []
    for o in old:
        w = max(1, case["nodes"] - rng.randrange(1 + case["nodes"] // 4))
        parents = _tree(rng, w, case["branch"])
        seqs.append((o, w, parents, _path(rng, parents)))
    return seqs


def _ancestors(parents):
    """Per drafted token the drafted tokens that it sees, itself among them, as bits."""
    bits = []
    for i, p in enumerate(parents):
        bits.append(1 << i | (bits[p] if p >= 0 else 0))
    return bits


def work(case):
    s, kind = Spec(case["model"]), case["kind"]
    seqs = _layout(case)
    if kind == "draft":
        new = sum(w for _, w, _, _ in seqs)
        moved = sum(j != x for _, _, _, path in seqs for j, x in enumerate(path))
        blocks = sum(_blocks(w) for _, w, _, _ in seqs)
        nbytes = new * 2 * (s.hq + s.hkv) * s.d * 2 + s.kv_bytes(new, blocks) + s.kv_bytes(2 * moved, 0)
        back = sum(len(path) for _, _, _, path in seqs)
        if s.e4m3:
            nbytes += s.kv_bytes(back, blocks) + back * s.hkv * s.d * 4
        return {"bytes": case["layers"] * nbytes, "flops": case["layers"] * 10 * new * (s.hq + s.hkv) * s.d}
    nbytes = seen = rows = 0
    for o, w, parents, _ in seqs:
        # tokens of the context that some query sees, and tokens seen by all queries together
        window = case["window"] or o + w
        lo = max(0, o + 1 - window)
        some = o + w - max(0, lo - min(case["sinks"], lo))
        nbytes += s.kv_bytes(some, _blocks(some))
        rows += w
        if kind == "tree":
            bits = _ancestors(parents)
            nbytes += 8 * len(bits) * ((case["nodes"] + 63) // 64)
            for b in bits:
                depth = bin(b).count("1")
                first = max(0, o + depth - window)
                seen += depth + o - first + min(case["sinks"], first)
        else:
            for p in range(o, o + w):
                first = max(0, p + 1 - window)
                seen += p + 1 - first + min(case["sinks"], first)
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


def _open(st, s, lens, layers=1, one_block_frames=False, seed=0):
    """A pool with one model whose rows 0, 1, ... have room for so many tokens.  With frames of one block handed out in order, row by
    row, the rows' blocks lie side by side in the pool; otherwise rows grow side by side on scattered frames."""
    from paper_2505_04021_amd import PKV_BF16, PKV_E4M3, PrismKV
    be = st.be = PrismKV(DEV)
    block = layers * (2 * T * s.hkv * s.d * (1 if s.e4m3 else 2) + (128 if s.e4m3 else 0))
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
    m = st.m = be.model_register(st.pool, s.hq, s.hkv, s.d, PKV_E4M3 if s.e4m3 else PKV_BF16, len(lens), st.max_blocks, layers)
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
    (k, ks), (v, vs) = cache
    b = _blocks(n)
    rows = [x[i, :b].reshape(b * T, s.hkv, s.d)[:n].contiguous().view(torch.uint8 if s.e4m3 else torch.int16) for x in (k, v)]
    assert st.be.kv_write(st.m, row, 0, rows[0], rows[1], ks[i, :b] if s.e4m3 else None, vs[i, :b] if s.e4m3 else None) == n


def _words(bits, words):
    """Masks as rows of 64-bit words (int64 holds the bits)."""
    return np.array([[(b >> 64 * w) & ((1 << 64) - 1) for w in range(words)] for b in bits], dtype=np.uint64).view(np.int64)


def prepare(case, seed):
    s, kind, g = Spec(case["model"]), case["kind"], _gen(seed)
    st = State()
    st.case, st.s = case, s
    seqs = _deal(seed, _layout(case))
    n = len(seqs)
    st.old, st.new = [x[0] for x in seqs], [x[1] for x in seqs]
    st.held = [o + w for o, w in zip(st.old, st.new)]
    st.ctx, st.q_lens = _i32(st.held), np.array(st.new, dtype=np.int32)
    rows, longest = sum(st.new), max(st.new)
    if kind in ("tree", "draft"):
        bits = [_ancestors(x[2]) for x in seqs]
        st.sees = torch.from_numpy(_words(sum(bits, []), (case["nodes"] + 63) // 64)).to(DEV)
        st.depth = torch.tensor([bin(b).count("1") - 1 for x in bits for b in x], device=DEV)
        st.bits = bits
    if kind == "draft":
        st.paths = [x[3] for x in seqs]
        st.kept_lens = [len(x) for x in st.paths]
        kept = np.zeros(rows, dtype=np.int32)
        first = np.cumsum([0] + st.new)
        for i, x in enumerate(st.paths):
            kept[first[i]:first[i] + len(x)] = x
        st.kept, st.n_kept = torch.from_numpy(kept).to(DEV), _i32(st.kept_lens)
        fused = _randn((case["layers"], rows, s.hq + 2 * s.hkv, s.d), g)
        st.q, st.k, st.v = fused[:, :, :s.hq], fused[:, :, s.hq:s.hq + s.hkv], fused[:, :, s.hq + s.hkv:]
        st.qw, st.kw = ((1.0 + 0.2 * _randn((s.d,), g).float()).to(torch.bfloat16) for _ in range(2)) if case["norm"] else (None, None)
        st.before = _i32([37 * i for i in range(n)])
        st.freq = 10000.0 ** (-torch.arange(case["rot"] // 2, dtype=torch.float64) / (case["rot"] // 2))
        if own:
            from paper_2505_04021_amd import PrismKV, ROTARY_HALF, ROTARY_PAIRS
            st.rotary = PrismKV(DEV).rotary_create(case["rot"], ROTARY_HALF if case["layout"] == "half" else ROTARY_PAIRS, st.freq.numpy())
            assert st.rotary >= 0
            _open(st, s, st.held, case["layers"], one_block_frames=not s.e4m3)
            st.q_out = torch.empty((case["layers"], rows, s.hq, s.d), dtype=torch.bfloat16, device=DEV)
            st.new_lens = torch.empty(n, dtype=torch.int32, device=DEV)
            if s.e4m3:
                back = sum(st.kept_lens)
                st.k_back, st.v_back = (torch.empty((case["layers"], back, s.hkv, s.d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
                st.every, st.begin, st.count = (np.array(x, dtype=np.int32) for x in (range(n), st.old, st.kept_lens))
            else:
                # the pool's bytes by sequence, block, layer and token: no copy, a view of the blocks' own order of elements
                x = st.storage.view(torch.bfloat16).view(n, st.max_blocks, case["layers"], s.hkv, 2, T * s.d)
                st.k_view = x[..., 0, :].view(n, st.max_blocks, case["layers"], s.hkv, s.d // 8, T, 8).permute(2, 0, 1, 5, 3, 4, 6)
                st.v_view = x[..., 1, :].view(n, st.max_blocks, case["layers"], s.hkv, s.d // 32, 4, 16, 2, 4).permute(2, 0, 1, 5, 8, 3, 4, 7, 6)
        else:
            blocks = max(_blocks(x) for x in st.held)
            seq = torch.repeat_interleave(torch.arange(n), torch.tensor(st.new))
            index = torch.cat([torch.arange(o, o + w) for o, w in zip(st.old, st.new)])
            st.seq, st.index = seq.to(DEV), index.to(DEV)          # each row's sequence and its index in it: the plain form's plan
            st.to_seq = torch.repeat_interleave(torch.arange(n), torch.tensor(st.kept_lens)).to(DEV)
            st.to_index = torch.tensor([o + j for o, x in zip(st.old, st.paths) for j in range(len(x))], device=DEV)
            st.from_index = torch.tensor([o + j for o, x in zip(st.old, st.paths) for j in x], device=DEV)
            st.base = torch.tensor(st.old, device=DEV)
            st.lens = torch.tensor(st.kept_lens, dtype=torch.int32, device=DEV)
            if not s.e4m3:
                st.k_cache, st.v_cache = (torch.zeros((case["layers"], n, blocks * T, s.hkv, s.d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return st
    st.q = _randn((rows, s.hq, s.d), g)
    cache = _cache(s, st.held, g)
    if own:
        _open(st, s, st.held, seed=seed)
        for i, x in enumerate(st.held):
            _fill(st, s, i, x, cache, i)
        st.out = torch.empty(st.q.shape, dtype=torch.float32, device=DEV)
        return st
    st.cache = cache
    st.first = torch.tensor(st.old, device=DEV)
    # ragged chunks as rows of equal length, a chunk's last token repeated, and the way back
    row0 = np.cumsum([0] + st.new)
    if kind == "window_prefill":
        longest = (longest + BAND - 1) // BAND * BAND if longest > BAND else longest
    st.rows = torch.tensor([[row0[i] + min(j, st.new[i] - 1) for j in range(longest)] for i in range(n)], device=DEV)
    st.back = torch.cat([torch.arange(w) + i * longest for i, w in enumerate(st.new)]).to(DEV)
    if kind == "tree":
        most = max(st.new)
        sees = np.zeros((rows, most), dtype=bool)
        for r, b in enumerate(sum(bits, [])):
            sees[r] = [b >> j & 1 for j in range(most)]
        st.seen_drafts = torch.from_numpy(sees).to(DEV)
    return st


# ---------------------------------------------------------------- one pass

def _values(cache):
    """Cached values in 32 bits, [n][tokens][Hkv][D]."""
    x, scale = cache
    y = x.float()
    if scale is not None:
        y = y * scale[:, :, None, :, None]
    return y.flatten(1, 2)


def _attend(q, k, v, seen):
    """softmax(q k^T) v over the tokens seen, 32 bits: q [..., rows, D], k and v [..., tokens, D], seen [..., rows, tokens]; zero rows where
    none is."""
    scores = torch.matmul(q, k.transpose(-1, -2)).masked_fill(~seen, -math.inf)
    m = scores.amax(dim=-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = torch.exp(scores - m)
    den = p.sum(dim=-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(den > 0, den, torch.ones_like(den))


def _plain_window(st):
    """Queries in blocks of at most BAND, each block with the band of tokens that its window covers and with the sinks."""
    s, c, n = st.s, st.case, len(st.new)
    q = st.q[st.rows].float() / math.sqrt(s.d)                    # [n][tokens][Hq][D]
    tokens = q.shape[1]
    band = min(BAND, tokens)
    blocks = tokens // band
    k, v = (_values(x) for x in st.cache)
    window, sinks = min(c["window"], k.shape[1]), min(c["sinks"], k.shape[1])
    at = st.first[:, None] + band * torch.arange(blocks, device=DEV)[None]          # [n][blocks]: position of a block's first query
    index = at[..., None] - window + 1 + torch.arange(window + band - 1, device=DEV)
    pos = (at[..., None] + torch.arange(band, device=DEV))[..., None]
    seen = (index[:, :, None] >= 0) & (index[:, :, None] <= pos) & (index[:, :, None] > pos - window)
    sink = torch.arange(sinks, device=DEV)
    seen = torch.cat([(sink <= pos - window), seen], dim=-1)                        # [n][blocks][band][sinks + window + band - 1]
    index = torch.cat([sink.expand(n, blocks, sinks), index.clamp(0, k.shape[1] - 1)], dim=-1)
    k, v = (x[torch.arange(n, device=DEV)[:, None, None], index].permute(0, 1, 3, 2, 4) for x in (k, v))
    q = q.view(n, blocks, band, s.hkv, s.g, s.d).permute(0, 1, 3, 2, 4, 5).reshape(n, blocks, s.hkv, band * s.g, s.d)
    out = _attend(q, k.contiguous(), v.contiguous(), seen.repeat_interleave(s.g, dim=2)[:, :, None])
    out = out.view(n, blocks, s.hkv, band, s.g, s.d).permute(0, 1, 3, 2, 4, 5).reshape(n * tokens, s.hq, s.d)
    return out[st.back]


def _plain_tree(st):
    s, c, n = st.s, st.case, len(st.new)
    q = st.q[st.rows].float() / math.sqrt(s.d)
    tokens = q.shape[1]
    k, v = (_values(x).permute(0, 2, 1, 3).contiguous() for x in st.cache)
    t = torch.arange(k.shape[2], device=DEV)
    base = st.first[:, None, None]
    seen = (t < base).expand(n, tokens, -1)
    if c["window"]:
        pos = base + st.depth[st.rows][..., None]
        seen = seen & ((t > pos - c["window"]) | (t < c["sinks"]))
    drafted = t - base                                             # [n][1][context]
    most = st.seen_drafts.shape[1]
    inside = (drafted >= 0) & (drafted < most)
    mine = torch.gather(st.seen_drafts[st.rows], 2, drafted.clamp(0, most - 1).expand(n, tokens, -1))
    seen = seen | (inside & mine)
    q = q.view(n, tokens, s.hkv, s.g, s.d).permute(0, 2, 1, 3, 4).reshape(n, s.hkv, tokens * s.g, s.d)
    out = _attend(q, k, v, seen.repeat_interleave(s.g, dim=1)[:, None])
    out = out.view(n, s.hkv, tokens, s.g, s.d).permute(0, 2, 1, 3, 4).reshape(n * tokens, s.hq, s.d)
    return out[st.back]


def _turned(x, weight, st):
    """x [layers][rows][heads][D] normed, if there is a weight, and rotated: 32 bits, angles in 64."""
    c = st.case
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + EPS) * weight.float()
    pos = st.before.double()[st.seq] + st.base.double()[st.seq] + st.depth.double()
    angle = pos[:, None] * st.freq.to(DEV)
    cos, sin = (f(angle).float()[:, None, :] for f in (torch.cos, torch.sin))
    r = c["rot"]
    if c["layout"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., r:]], dim=-1).to(torch.bfloat16)
    a, b = y[..., 0:r:2], y[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2), y[..., r:]], dim=-1).to(torch.bfloat16)


def _encode(v):
    return v.clamp(-E4M3_MAX, E4M3_MAX).to(E4M3).float()


def _append_blocks(y, there, stays, codes0, scale0):
    """What blocks hold after the tokens y [blocks][T][Hkv][D] (those that are `there`) have been appended one after the other: one scale for a
    block and kv head, the largest amax / 448 so far; where a token raises it, the codes before are encoded again.  Tokens that `stay` are
    in place already, with codes0 and scale0."""
    cand = y.abs().amax(dim=-1) / torch.full((), E4M3_MAX, device=DEV)             # (a number would be a product with its reciprocal)
    first = torch.where(cand[:, 0] > 0, cand[:, 0], torch.ones_like(cand[:, 0]))
    scale = torch.where(stays[:, 0, None], scale0, first)
    codes = torch.zeros_like(y)
    for t in range(T):
        up = torch.where((there[:, t] & ~stays[:, t])[:, None], torch.maximum(scale, cand[:, t]), scale)
        codes = torch.where((up > scale)[:, None, :, None], _encode(codes * scale[:, None, :, None] / up[:, None, :, None]), codes)
        scale = up
        mine = torch.where(stays[:, t, None, None], codes0[:, t], _encode(y[:, t] / scale[:, :, None]))
        codes[:, t] = torch.where(there[:, t, None, None], mine, codes[:, t])
    return codes, scale


def _kept_codes(x, st):
    """What an e4m3 cache gives back of the accepted tokens, after rows x [layers][rows][Hkv][D] were appended and those tokens moved together."""
    s, n, layers = st.s, len(st.new), x.shape[0]
    blocks = max(_blocks(w) for w in st.new)
    shape = (layers, n, blocks * T, s.hkv, s.d)
    local = st.index - st.base[st.seq]                             # (drafts begin a block)
    y = torch.zeros(shape, device=DEV)
    y[:, st.seq, local] = x.float()
    there = torch.zeros((layers, n, blocks * T), dtype=torch.bool, device=DEV)
    there[:, st.seq, local] = True
    view = lambda z: z.view(layers * n * blocks, T, *z.shape[3:])  # noqa: E731
    none = torch.zeros_like(view(there))
    codes, scale = _append_blocks(view(y), view(there), none, view(y), torch.ones((layers * n * blocks, s.hkv), device=DEV))
    back = (codes * scale[:, None, :, None]).view(shape).to(torch.bfloat16).float()
    # the accepted tokens, those at the front that do not move aside
    to, frm = st.to_index - st.base[st.to_seq], st.from_index - st.base[st.to_seq]
    y2 = torch.zeros(shape, device=DEV)
    y2[:, st.to_seq, to] = back[:, st.to_seq, frm]
    there2, stays = torch.zeros_like(there), torch.zeros_like(there)
    there2[:, st.to_seq, to] = True
    stays[:, st.to_seq, to] = to == frm
    codes, scale = _append_blocks(view(y2), view(there2), view(stays), codes, scale)
    back = (codes * scale[:, None, :, None]).view(shape)
    return back[:, st.to_seq, to].to(torch.bfloat16)


def run(st):
    c, s, kind = st.case, st.s, st.case["kind"]
    if own:
        be, m = st.be, st.m
        if kind == "window_decode":
            be.decode_attention_window_dev(m, st.q, st.ctx, c["window"], c["sinks"], st.out)
        elif kind == "window_prefill":
            be.prefill_attention_window_dev(m, st.q, st.q_lens, st.ctx, c["window"], c["sinks"], st.out)
        elif kind == "tree":
            be.tree_attention_dev(m, st.q, st.q_lens, st.ctx, st.sees, st.out, c["window"], c["sinks"])
        else:
            for layer in range(c["layers"]):
                be.set_layer(m, layer)
                be.qkv_append_tree_dev(m, st.q[layer], st.k[layer], st.v[layer], st.q_lens, st.ctx, st.sees, st.q_out[layer], st.qw, st.kw, EPS, st.rotary, st.before)
            be.kv_keep_dev(m, st.q_lens, st.ctx, st.kept, st.n_kept, st.new_lens)
            if s.e4m3:
                for layer in range(c["layers"]):
                    be.set_layer(m, layer)
                    be.kv_gather_dev(m, st.every, st.begin, st.count, st.k_back[layer], st.v_back[layer])
                return st.q_out, st.k_back, st.v_back, st.new_lens
            return st.q_out, st.k_view, st.v_view, st.new_lens
        return st.out
    if kind in ("window_decode", "window_prefill"):
        return _plain_window(st)
    if kind == "tree":
        return _plain_tree(st)
    q, k = _turned(st.q, st.qw, st), _turned(st.k, st.kw, st)
    lens = (st.base + st.lens).to(torch.int32)
    if s.e4m3:
        return q, _kept_codes(k, st), _kept_codes(st.v, st), lens
    for cache, x in ((st.k_cache, k), (st.v_cache, st.v)):
        cache[:, st.seq, st.index] = x
        cache[:, st.to_seq, st.to_index] = cache[:, st.to_seq, st.from_index]
    layers, n = c["layers"], len(st.new)
    return q, st.k_cache.view(layers, n, -1, T, s.hkv, s.d // 8, 8), st.v_cache.view(layers, n, -1, 4, 4, s.hkv, s.d // 32, 2, 16), lens


# ---------------------------------------------------------------- the same in 64 bits

def _exact_turn(row, weight, pos, freq, case):
    """Heads [..., heads][D] in 64 bits, element pairs as complex numbers."""
    y = row.double()
    if weight is not None:
        y = weight.double() * y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / y.shape[-1] + EPS)
    r, h = case["rot"], case["rot"] // 2
    first, second = (y[..., :h], y[..., h:r]) if case["layout"] == "half" else (y[..., 0:r:2], y[..., 1:r:2])
    z = torch.complex(first, second) * torch.polar(torch.ones_like(freq), freq * pos)
    y = y.clone()
    if case["layout"] == "half":
        y[..., :h], y[..., h:r] = z.real, z.imag
    else:
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    return y


def _exact_append(held, scale, x):
    """A block's e4m3 values [tokens][Hkv][D] and scale after one more token x [Hkv][D]; held is None for an empty block."""
    rnd = lambda v: v.float().clamp(-E4M3_MAX, E4M3_MAX).to(E4M3).float()  # noqa: E731
    x = x.float()
    cand = x.abs().amax(-1, keepdim=True) / torch.tensor(E4M3_MAX, device=DEV)
    if held is None:
        scale = torch.where(cand > 0, cand, torch.ones_like(cand))
        return rnd(x / scale)[None], scale
    up = torch.maximum(cand, scale)
    held = torch.where(up > scale, rnd(held * scale / up), held)
    return torch.cat([held, rnd(x / up)[None]]), up


def _exact_kept(rows, path):
    """Accepted tokens of one sequence and layer as an e4m3 cache holds them, drafted rows [tokens][Hkv][D] from the start of a block on."""
    blocks = []
    for b in range(0, len(rows), T):
        held = scale = None
        for x in rows[b:b + T]:
            held, scale = _exact_append(held, scale, x)
        blocks.append((held, scale))
    value = lambda i: (blocks[i // T][0][i % T] * blocks[i // T][1]).to(torch.bfloat16)  # noqa: E731
    moved = [value(i) for i in path]
    done = []
    for b in range(0, len(path), T):
        some = path[b:b + T]
        stay = sum(i == b + j for j, i in enumerate(some))
        held, scale = (blocks[b // T][0][:stay], blocks[b // T][1]) if stay else (None, None)
        for j in range(stay, len(some)):
            held, scale = _exact_append(held, scale, moved[b + j])
        done.append(held.double() * scale.double())
    return torch.cat(done)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    s, kind = st.s, case["kind"]
    row0 = np.cumsum([0] + st.new)
    if kind == "draft":
        if s.e4m3 and case["layers"] * sum(st.new) > 600:
            return None
        pos = torch.tensor([37 * i + st.old[i] + bin(b).count("1") - 1 for i, x in enumerate(st.bits) for b in x], device=DEV).double()[:, None, None]
        q, k = (_exact_turn(x, w, pos, st.freq.to(DEV), case) for x, w in ((st.q, st.qw), (st.k, st.kw)))
        lens = torch.tensor([o + len(x) for o, x in zip(st.old, st.paths)], dtype=torch.int32, device=DEV)
        if s.e4m3:
            back = [torch.stack([torch.cat([_exact_kept(x[layer, row0[i]:row0[i + 1]], st.paths[i]) for i in range(len(st.new))])
                                 for layer in range(case["layers"])]) for x in (k.to(torch.bfloat16), st.v)]
            return q, back[0], back[1], lens
        caches = []
        for x in (k, st.v.double()):
            c = torch.zeros((case["layers"], len(st.new), max(_blocks(h) for h in st.held) * T, s.hkv, s.d), dtype=torch.float64, device=DEV)
            for i, path in enumerate(st.paths):
                rows = x[:, row0[i]:row0[i + 1]]
                c[:, i, st.old[i]:st.held[i]] = rows
                c[:, i, st.old[i]:st.old[i] + len(path)] = rows[:, path]
            caches.append(c)
        return (q, caches[0].reshape(case["layers"], len(st.new), -1, T, s.hkv, s.d // 8, 8),
                caches[1].reshape(case["layers"], len(st.new), -1, 4, 4, s.hkv, s.d // 32, 2, 16), lens)
    answers = []
    for i, (o, w) in enumerate(zip(st.old, st.new)):
        k, v = ((x[0][i].double() * (x[1][i].double()[:, None, :, None] if x[1] is not None else 1.0)).flatten(0, 1)[:o + w] for x in st.cache)
        t = np.arange(o + w)
        may = np.zeros((w, o + w), dtype=bool)
        for j in range(w):
            if kind == "tree":
                b = st.bits[i][j]
                p = o + bin(b).count("1") - 1
                may[j] = (t < o) & ((t > p - case["window"]) | (t < case["sinks"]) | (case["window"] == 0))
                may[j, o:] = [bool(b >> x & 1) for x in range(w)]
            else:
                may[j] = (t <= o + j) & ((t > o + j - case["window"]) | (t < case["sinks"]))
        hidden = torch.from_numpy(~may).to(DEV)
        out = torch.zeros((w, s.hq, s.d), dtype=torch.float64, device=DEV)
        for h in range(s.hq):
            z = st.q[row0[i]:row0[i + 1], h].double() @ k[:, h // s.g].t().contiguous() * s.d ** -0.5
            out[:, h] = torch.softmax(z.masked_fill(hidden, -math.inf), dim=-1) @ v[:, h // s.g].contiguous()
        answers.append(out)
    return torch.cat(answers)
