"""Operators over a long key/value cache that a pass should not have to read whole, as cases that can be prepared, run and timed.

  window   glance_attention with a sliding window: every row sees the first `sinks` positions and the last `window` ones
           (its own among them) of a paged bf16 cache.
  packed   glance_attention over a mixed cache: whole pages of committed context held in 4 bits, the rest in bf16;
           with or without a window.
  pack     glance_pack_cache and glance_unpack_cache: whole pages of committed context of every layer into the 4-bit
           pool, and the values that they stand for back into a bf16 pool.

The rows of a pass are single tokens ("token"), the nodes of a candidate tree ("tree"), a block whose rows all see each
other ("block") or a chain ("chain": a prefill pass).  Row i of a sequence with P committed positions stands at position
P + depth(i), which is P + i in a block or a chain; its key and value lie in the cache at row P + i.  It sees committed
position p if p < sinks or P + depth(i) - p < window, and row j if the tree, block or chain lets it and likewise
P + depth(j) < sinks or depth(i) - depth(j) < window.  window 0 means no limit.

The 4-bit format: 16 values along the head dimension share a scale s, the e4m3 value nearest to max|x| / 6; a value is s
times the e2m1 value (0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign) nearest to x / s; ties go to the even code.

Head layouts are the repository's own (tiny, small, 7b) and generic ones; lengths reach from one position to documents.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE, GROUP = 64, 16
# query heads, kv heads, head dimension
HEADS = {"tiny": (4, 2, 64), "small": (16, 4, 64), "7b": (28, 4, 128), "32/8": (32, 8, 128), "8/8": (8, 8, 128), "16/1": (16, 1, 64)}


def listed():
    return [
        # plain decoding of one short sequence behind a window: the smallest call, all latency
        dict(name="window-token", kind="window", heads="7b", rows="token", T=1, lo=1536, hi=1536, batch=1, window=512, sinks=4),
        # plain decoding of eight documents, a window over each and the first page of the image kept
        dict(name="window-token-batch", kind="window", heads="7b", rows="token", T=1, lo=2500, hi=8704, batch=8, window=2000, sinks=64),
        # the widest candidate tree over a document-sized image prefix
        dict(name="window-tree", kind="window", heads="7b", rows="tree", T=128, lo=8704, hi=8704, batch=1, window=2048, sinks=256),
        # a prefill pass of a long prompt, odd in every size
        dict(name="window-chain", kind="window", heads="7b", rows="chain", T=1999, lo=4133, hi=4133, batch=1, window=1000, sinks=5),
        # plain decoding of one long document
        dict(name="packed-token-long", kind="packed", heads="7b", rows="token", T=1, lo=32801, hi=32801, batch=1, window=0, sinks=0, tail=64),
        # plain decoding of a batch of ragged documents
        dict(name="packed-token-batch", kind="packed", heads="7b", rows="token", T=1, lo=4096, hi=32768, batch=16, window=0, sinks=0, tail=200),
        # the benchmark's tree over a document-sized image prefix
        dict(name="packed-tree", kind="packed", heads="7b", rows="tree", T=64, lo=8704, hi=8704, batch=1, window=0, sinks=0, tail=64),
        # small-batch serving: trees of eight ragged sequences
        dict(name="packed-tree-batch", kind="packed", heads="7b", rows="tree", T=64, lo=1024, hi=4096, batch=8, window=0, sinks=0, tail=64),
        # a draft block of the small model over a 4-bit context with a window
        dict(name="packed-window-block", kind="packed", heads="small", rows="block", T=8, lo=5003, hi=5003, batch=2, window=1500, sinks=70, tail=100),
        # one finished page of every layer: what a round of a running sequence adds
        dict(name="pack-page", kind="pack", heads="7b", layers=28, lo=64, hi=127, batch=1, tail=0),
        # ragged contexts of the small model
        dict(name="pack-ragged", kind="pack", heads="small", layers=8, lo=300, hi=1900, batch=5, tail=33),
        # a document's context after its prefill
        dict(name="pack-context", kind="pack", heads="7b", layers=28, lo=8704, hi=8704, batch=1, tail=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["window", "window", "packed", "packed", "packed", "pack"])
    heads = rng.choice(list(HEADS))
    if kind == "pack":
        batch = rng.randint(1, 6)
        tail = rng.choice([0, 0, 1, 64, 200])
        lo = max(_log_int(rng, 64, 8000 // batch), PAGE + tail)
        return dict(kind=kind, heads=heads, layers=_log_int(rng, 1, 16), lo=lo, hi=lo + rng.choice([0, lo // 3]), batch=batch, tail=tail)
    rows = rng.choice(["token", "token", "tree", "tree", "block", "chain"])
    batch = rng.choice([1, 1, 1, 2, 5, 8, 16])
    if rows == "chain":
        batch, T = 1, _log_int(rng, 2, 1900)
    else:
        T = 1 if rows == "token" else _log_int(rng, 2, 128 if rows == "tree" else 16)
    lo = _log_int(rng, 1, min(32768, 4500 if rows == "chain" else 200000 // batch if T == 1 else 8704 if batch <= 2 else 2048))
    window = _log_int(rng, 1, 4096) if kind == "window" or rng.random() < 0.3 else 0
    case = dict(kind=kind, heads=heads, rows=rows, T=T, lo=lo, hi=lo + (rng.choice([0, lo // 4]) if batch > 1 else 0), batch=batch, window=window,
                sinks=rng.choice([0, 1, 4, 64, rng.randint(2, 500)]) if window else 0)
    if kind == "packed":
        case["tail"] = rng.choice([0, 1, 64, rng.randint(2, 400)])
    return case


# ---- inputs --------------------------------------------------------------------------------------------------------
def _lengths(c):
    """Committed positions of every sequence: the case's, whatever the seed."""
    return [int(v) for v in np.random.default_rng((c["lo"], c["hi"], 1)).integers(c["lo"], c["hi"] + 1, size=c["batch"])]


def _held(c, P):
    """Positions held in 4 bits: whole pages, at least `tail` positions left in bf16."""
    return max(0, P - c["tail"]) // PAGE * PAGE if "tail" in c else 0


def _parents(c, seed):
    """Parents [batch][T] of the rows (-1: sees itself only), in an order in which parents come first."""
    rng = np.random.default_rng((seed, 7))
    T, out = c["T"], np.full((c["batch"], c["T"]), -1, dtype=np.int64)
    for s in range(c["batch"]):
        nodes = T - (int(rng.integers(0, T // 8 + 1)) if T > 8 else 0)     # the last rows may be padding
        for i in range(1, nodes):
            out[s, i] = i - 1 if rng.random() < 0.5 else int(rng.integers(max(0, i - 12), i))
    return out


def _depths(parents):
    depth = np.zeros_like(parents)
    for s in range(parents.shape[0]):
        for i in range(parents.shape[1]):
            if parents[s, i] >= 0:
                depth[s, i] = depth[s, parents[s, i]] + 1
    return depth


def _ancestors(parents):
    """Truth values [batch][T][T]: column j is row i itself or an ancestor of it."""
    batch, T = parents.shape
    see = np.zeros((batch, T, T), dtype=bool)
    for s in range(batch):
        for i in range(T):
            if parents[s, i] >= 0:
                see[s, i] = see[s, parents[s, i]]
            see[s, i, i] = True
    return see


def _drawn(c, seed):
    """Pages of the cache and queries, from the seed alone.  Keys have louder and quieter channels, as projections give them."""
    Hq, Hkv, d = HEADS[c["heads"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens = _lengths(c)
    T, layers = c.get("T", 0), c.get("layers", 1)
    pages = (max(lens) + T + PAGE - 1) // PAGE
    table = torch.randperm(c["batch"] * pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32).view(c["batch"], pages)
    pool = torch.empty(layers, c["batch"] * pages, 2, Hkv, PAGE, d, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=gen)
    pool[:, :, 0] *= torch.exp(0.5 * torch.randn(Hkv, 1, d, device="cuda", generator=gen)).to(torch.bfloat16)
    q = torch.randn(c["batch"] * T, Hq * d, device="cuda", generator=gen).to(torch.bfloat16) if T else None
    return lens, table, pool, q


def prepare(case, seed):
    c = case
    lens, table, pool, q = _drawn(c, seed)
    state = dict(case=c, lens=lens, q=q)
    held = [_held(c, P) for P in lens]
    parents = _parents(c, seed) if c["kind"] != "pack" and c["rows"] == "tree" else None
    if own:
        return _prepare_own(state, table, pool, held, parents)
    state["pool"], state["table"] = pool, table.long().cuda()
    if parents is not None:
        state["see"] = torch.from_numpy(_ancestors(parents)).cuda()
        state["depth"] = torch.from_numpy(_depths(parents)).cuda()
    if c["kind"] == "packed":
        # the 4-bit part of the cache as codes (two to a byte) and e4m3 scales, one tensor of each per sequence: [2][Hkv][held][...]
        state["held"] = []
        for s, n in enumerate(held):
            rows = pool[0, state["table"][s, : n // PAGE]].permute(1, 2, 0, 3, 4).reshape(2, pool.shape[3], n, pool.shape[5])
            code, scale = _quantise(rows.float())
            state["held"].append((code[..., 0::2] | code[..., 1::2] << 4, scale))
    return state


def _prepare_own(state, table, pool, held, parents):
    """An engine whose cache holds these pages.  The operators read no weights, so the model around the heads is as small as it gets."""
    from paper_2609_00355_b200 import binding, synth
    c = state["case"]
    Hq, Hkv, d = HEADS[c["heads"]]
    H = 64
    cfg = synth.RoundConfig(name="case", n_layers=pool.shape[0], hidden=H, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, ffn=64, vocab=64, n_img=0, n_txt=0,
                            block_B=16, topk=1, tree_N=128, p_m=0.8, rounds=1, batch=c["batch"])
    zeros = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")
    layer = dict(ln1=zeros(H), wqkv=zeros((Hq + 2 * Hkv) * d, H), wo=zeros(H, Hq * d), ln2=zeros(H), wgu=zeros(128, H), wd=zeros(H, 64))
    target = dict(embed=zeros(64, H), lm_head=zeros(64, H), final_norm=zeros(H), layers=[layer] * cfg.n_layers)
    head = dict(layer, mask_embed=zeros(H), ctx_norm=zeros(H), final_norm=zeros(H))
    eng = binding.Engine(cfg, target, head, batch=c["batch"], max_len=table.shape[1] * PAGE)
    eng.page_table.copy_(table)
    eng.kv_pool.copy_(pool)
    eng.seq_len.copy_(torch.tensor(state["lens"], dtype=torch.int32))
    state["eng"] = eng
    if c["kind"] != "pack":
        state["out"] = torch.zeros_like(state["q"])
        if parents is not None:
            see, W = _ancestors(parents), (c["T"] + 63) // 64
            words = np.zeros((c["batch"], c["T"], W), dtype=np.uint64)
            for j in range(c["T"]):
                words[:, :, j // 64] |= see[:, :, j].astype(np.uint64) << np.uint64(j % 64)
            state["anc"] = torch.from_numpy(words.view(np.int64)).cuda()
    if c["kind"] != "window":
        eng.glance_set_packed(binding.PackedCache(eng))
        if c["kind"] == "packed":
            eng.glance_pack_cache(keep=c["tail"])
        else:
            state["none"] = torch.zeros_like(eng.seq_len)
            state["back"] = torch.zeros_like(eng.kv_pool)
    torch.cuda.synchronize()
    return state


# ---- one pass ------------------------------------------------------------------------------------------------------
def run(state):
    c = state["case"]
    if own:
        eng = state["eng"]
        if c["kind"] == "pack":
            eng.glance_pack_cache(keep=c["tail"])
            eng.glance_unpack_cache(state["none"], kv_pool=state["back"])
            return state["back"]
        eng.glance_attention(0, state["q"], c["T"], state["out"], anc=state.get("anc"), causal=c["rows"] == "chain", window=c["window"], sinks=c["sinks"])
        return state["out"]
    return _plain_pack(state) if c["kind"] == "pack" else _plain_attention(state)


def _quantise(x):
    """Codes (sign in bit 3) and e4m3 scales of groups of 16 along the last axis."""
    g = x.unflatten(-1, (-1, GROUP))
    scale = (g.abs().amax(-1, keepdim=True) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = scale.float()
    m = torch.where(s > 0, g.abs() / s, 0.0)
    # the borders between neighbouring magnitudes; a tie goes to the even code
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)).to(torch.uint8)
    code |= torch.signbit(g).to(torch.uint8) << 3
    return code.flatten(-2), scale.squeeze(-1)


def _values(code, scale):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    v = table[(code & 7).int()]
    v = torch.where(code >= 8, -v, v)
    return (v.unflatten(-1, (-1, GROUP)) * scale.float().unsqueeze(-1)).flatten(-2)


def _plain_pack(state):
    c, pool = state["case"], state["pool"]
    back = torch.zeros_like(pool)
    for s, P in enumerate(state["lens"]):
        ids = state["table"][s, : _held(c, P) // PAGE]
        back[:, ids] = _values(*_quantise(pool[:, ids].float())).to(torch.bfloat16)
    return back


def _plain_attention(state):
    c = state["case"]
    Hq, Hkv, d = HEADS[c["heads"]]
    T, G, window, sinks = c["T"], Hq // Hkv, c["window"], c["sinks"]
    out = torch.empty_like(state["q"])
    dev = out.device
    row = torch.arange(T, device=dev)
    for s, P in enumerate(state["lens"]):
        depth = state["depth"][s] if "depth" in state else row
        # positions that some row sees
        first = max(0, P - window + 1) if window else 0
        pos = torch.arange(P + T, device=dev) if first <= sinks else torch.cat([torch.arange(sinks, device=dev), torch.arange(first, P + T, device=dev)])
        held = _held(c, P)
        kv = state["pool"][0][state["table"][s, pos // PAGE], :, :, pos % PAGE].float().permute(1, 2, 0, 3)      # [2][Hkv][keys][d]
        if held:
            packed, scale = state["held"][s]
            at = pos[pos < held]
            b = packed[:, :, at]
            code = torch.stack([b & 15, b >> 4], -1).flatten(-2)
            kv = torch.cat([_values(code, scale[:, :, at]), kv[:, :, at.numel():]], 2)
        q = state["q"][s * T : (s + 1) * T].float().view(T, Hkv, G, d).permute(1, 2, 0, 3).reshape(Hkv, G * T, d)
        at_row = P + depth                                                                                      # position of every row
        new = pos >= P
        at_key = torch.where(new, P + depth[(pos - P).clamp(min=0)], pos)
        if "see" in state:
            seen = state["see"][s][:, (pos - P).clamp(min=0)] | ~new
        elif c["rows"] == "chain":
            seen = at_key <= at_row[:, None]
        else:
            seen = torch.ones(T, pos.numel(), dtype=torch.bool, device=dev)
        if window:
            seen = seen & ((at_key < sinks) | (at_row[:, None] - at_key < window))
        x = (q @ kv[0].transpose(1, 2)) * (d ** -0.5)
        x = x.view(Hkv, G, T, -1).masked_fill_(~seen, -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        x = x / x.sum(-1, keepdim=True)
        y = x.view(Hkv, G * T, -1) @ kv[1]
        out[s * T : (s + 1) * T] = y.view(Hkv, G, T, d).permute(2, 0, 1, 3).reshape(T, Hq * d).to(torch.bfloat16)
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def work(case):
    c = case
    Hq, Hkv, d = HEADS[c["heads"]]
    row16, row4 = 2 * Hkv * d * 2, 2 * Hkv * (d // 2 + d // GROUP)       # bytes of a position: K and V of all kv heads
    if c["kind"] == "pack":
        n = c["layers"] * sum(_held(c, P) for P in _lengths(c))
        return {"bytes": n * (2 * row16 + 2 * row4), "flops": 4 * n * 2 * Hkv * d}
    T, pairs, total = c["T"], 0, 0
    depth = _depths(_parents(c, 0)) if c["rows"] == "tree" else np.tile(np.arange(T), (c["batch"], 1))
    for s, P in enumerate(_lengths(c)):
        held = _held(c, P)
        for k, dep in enumerate(depth[s].tolist()):
            first = max(0, P + dep - c["window"] + 1) if c["window"] else 0
            pairs += max(0, P - first) + min(first, c["sinks"], P)
            pairs += T if c["rows"] == "block" else min(dep + 1, c["window"] or dep + 1)
        first = max(0, P - c["window"] + 1) if c["window"] else 0
        first = max(first, min(c["sinks"], P))
        total += (max(0, held - first) + min(held, first, c["sinks"])) * row4
        total += (max(0, P - max(first, held)) + max(0, min(first, c["sinks"]) - held) + T) * row16
    return {"bytes": total + 2 * c["batch"] * T * Hq * d * 2, "flops": 4 * d * Hq * pairs}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------
def _held_values(x):
    """The 64-bit values that groups of 16 of x are held as."""
    g = x.reshape(-1, GROUP)
    a = g.abs().max(1).values / 6
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(a, min=2.0 ** -40))), min=-6.0) - 3)
    s = torch.clamp(torch.round(a / step) * step, max=448.0)[:, None]
    m = torch.where(s > 0, g.abs() / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(g))
    unit = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).double()
    return (torch.copysign(torch.clamp(torch.round(m / unit) * unit, max=6.0), g) * s).reshape(x.shape)


def exact(case, seed):
    c = case
    Hq, Hkv, d = HEADS[c["heads"]]
    lens, table, pool, q = _drawn(c, seed)
    table = table.cuda().long()
    if c["kind"] == "pack":
        out = torch.zeros(pool.shape, dtype=torch.float64, device="cuda")
        for s, P in enumerate(lens):
            for p in table[s, : _held(c, P) // PAGE].tolist():
                out[:, p] = _held_values(pool[:, p].double())
        return out
    T = c["T"]
    depth = None
    if c["rows"] == "tree":
        parents = _parents(c, seed)
        depth = _depths(parents)
    out = torch.empty(c["batch"] * T, Hq * d, dtype=torch.float64, device="cuda")
    for s, P in enumerate(lens):
        rows = pool[0, table[s]].permute(1, 2, 0, 3, 4).reshape(2, Hkv, -1, d)[:, :, : P + T].double()
        n = _held(c, P)
        if n:
            rows[:, :, :n] = _held_values(rows[:, :, :n])
        at = np.arange(P + T, dtype=np.int64)
        if depth is not None:
            at[P:] = P + depth[s]
        seen = np.ones((T, P + T), dtype=bool)
        if c["rows"] == "tree":
            seen[:, P:] = False
            for i in range(T):
                j = i
                while j >= 0:
                    seen[i, P + j] = True
                    j = int(parents[s, j])
        elif c["rows"] == "chain":
            seen[:, P:] = np.tri(T, dtype=bool)
        if c["window"]:
            for i in range(T):
                seen[i] &= (at < c["sinks"]) | (at > at[P + i] - c["window"])
        hide = torch.from_numpy(~seen).cuda()
        for h in range(Hq):
            k, v = rows[0, h // (Hq // Hkv)], rows[1, h // (Hq // Hkv)]
            score = q[s * T : (s + 1) * T, h * d : (h + 1) * d].double() @ k.T / math.sqrt(d)
            out[s * T : (s + 1) * T, h * d : (h + 1) * d] = torch.softmax(score.masked_fill(hide, -math.inf), dim=1) @ v
    return out
