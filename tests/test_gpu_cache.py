"""Attention over a cache that is read in part (sliding window, sinks) or held in 4 bits, and the packing of that cache (GPU).

References are written from the definitions in 64 bits.  Tolerances, derived before the first run, with A = sum_j p_j |v_j|
(what the output would be without cancellation):
  * out is bf16: half a step, 2^-8 of the value;
  * probabilities are rounded to fp16 or to two terms: 2^-11 of A at most;
  * scores are fp32 sums of d products: (d + 2) 2^-24 sum |q||k| / sqrt(d), below 2 x 10^-4 for the inputs here (sum |q||k| /
    sqrt(d) < 13 on average over a row); numerator and denominator each carry it: less than 2^-11 of A together;
so |out - ref| <= 2^-8 |ref| + 2^-10 A.  With two-term queries and outputs (hi + lo: 2^-16) and two-term probabilities
(2^-16) only the scores' error stays: 2^-15 |ref| + 2^-11 A.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2609_00355_b200 import synth

PAGE, GROUP = 64, 16


# ---- definitions in 64 bits ----------------------------------------------------------------------------------------
def held_values(x):
    """What groups of 16 along the last axis are held as: e2m1 codes with an e4m3 scale, ties to the even code."""
    g = x.double().unflatten(-1, (-1, GROUP))
    a = g.abs().amax(-1, keepdim=True) / 6
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -40))).clamp(min=-6) - 3)
    s = (torch.round(a / step) * step).clamp(max=448)
    m = torch.where(s > 0, g.abs() / torch.where(s > 0, s, 1.0), 0.0)
    unit = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).double()
    v = torch.copysign((torch.round(m / unit) * unit).clamp(max=6), g) * s
    v = torch.where(torch.isfinite(g).all(-1, keepdim=True), v, math.nan)
    return v.flatten(-2)


def visible(P, T, kind, parents, window, sinks):
    """[T][P + T] truth values: which cache rows each row sees."""
    see = np.ones((T, P + T), dtype=bool)
    at = np.arange(P + T)
    if kind == "tree":
        see[:, P:] = False
        for i in range(T):
            j, chain = i, []
            while j >= 0:
                see[i, P + j] = True
                chain.append(j)
                j = int(parents[j])
            at[P + i] = P + len(chain) - 1
    elif kind == "chain":
        see[:, P:] = np.tri(T, dtype=bool)
    if window:
        for i in range(T):
            see[i] &= (at < sinks) | (at[P + i] - at < window)
    return see


def reference(q, K, V, see):
    """q [T][Hq][d], K, V [P + T][Hkv][d] float64 -> out [T][Hq][d] and A.  Rows that see nothing are zeros."""
    T, Hq, d = q.shape
    G = Hq // K.shape[1]
    see = torch.from_numpy(see).to(q.device)
    out, A = torch.zeros_like(q), torch.zeros_like(q)
    some = see.any(1)
    used = see.any(0)
    for h in range(Hq):
        k, v = K[used, h // G], V[used, h // G]
        s = (q[:, h] @ k.T / math.sqrt(d)).masked_fill(~see[:, used], -math.inf)
        p = torch.softmax(s[some], dim=1)
        out[some, h] = p @ v
        A[some, h] = p @ v.abs()
    return out, A


def random_parents(T, rng):
    parents = np.full(T, -1)
    nodes = T - (int(rng.integers(0, T // 8 + 1)) if T > 8 else 0)
    for i in range(1, nodes):
        parents[i] = i - 1 if rng.random() < 0.6 else int(rng.integers(max(0, i - 12), i))
    return parents


def anc_words(parents):
    T = len(parents)
    W = (T + 63) // 64
    words = np.zeros((T, W), dtype=np.uint64)
    for i in range(T):
        j = i
        while j >= 0:
            words[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
            j = int(parents[j])
    return words.view(np.int64)


# ---- engine whose cache is ours --------------------------------------------------------------------------------------
def make_engine(heads, batch, max_len, layers=1, stream=None):
    from paper_2609_00355_b200.binding import Engine
    Hq, Hkv, d = heads
    cfg = synth.RoundConfig(name="cache", n_layers=layers, hidden=64, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, ffn=64, vocab=64, n_img=0,
                            n_txt=0, block_B=16, topk=1, tree_N=128, p_m=0.8, rounds=1, batch=batch)
    tw, hw = synth.make_weights(cfg, "cuda")
    eng = Engine(cfg, tw, hw, batch=batch, max_len=max_len, stream=stream)
    return eng


class Cache:
    """An engine, random cache contents, and what they are in 64 bits."""

    def __init__(self, heads, lens, T, seed, held=None, layers=1, junk=True, stream=None):
        from paper_2609_00355_b200.binding import PackedCache
        self.heads, self.lens, self.T = heads, lens, T
        Hq, Hkv, d = heads
        batch = len(lens)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.eng = eng = make_engine(heads, batch, max(lens) + T, layers, stream)
        loud = torch.exp(0.5 * torch.randn(Hkv, 1, d, device="cuda", generator=g))
        pool = torch.randn(eng.kv_pool.shape, device="cuda", generator=g)
        pool[:, :, 0] *= loud
        eng.kv_pool.copy_(pool)
        eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        self.K, self.V = [], []
        for s, P in enumerate(lens):
            K, V = eng.gather_kv(s, 0, P + T)
            self.K.append(K.double())
            self.V.append(V.double())
        if junk:                                          # places beyond the last row hold anything
            for s, P in enumerate(lens):
                at = (P + T) % PAGE
                if at:
                    eng.kv_pool[:, int(eng.page_table[s, (P + T) // PAGE]), :, :, at:] = math.nan
        if held is not None:
            self.packed = PackedCache(eng)
            # (pages in an order of their own)
            self.packed.page_table.copy_(torch.randperm(batch * eng.pages_per_seq, generator=torch.Generator().manual_seed(seed)).to(torch.int32).view(batch, -1))
            eng.glance_set_packed(self.packed)
            eng.glance_pack_cache(keep=held)
            assert self.packed.len.tolist() == [max(0, P - held) // PAGE * PAGE for P in lens]
            for s, n in enumerate(self.packed.len.tolist()):
                self.K[s][:n] = held_values(self.K[s][:n])
                self.V[s][:n] = held_values(self.V[s][:n])
                for p in range(n // PAGE):                # the bf16 pages are not read any more
                    eng.kv_pool[:, int(eng.page_table[s, p])] = math.nan
            eng.page_table.copy_(torch.where(torch.arange(eng.pages_per_seq, device="cuda")[None] < self.packed.len[:, None] // PAGE, -7, eng.page_table))
        self.q = torch.randn(batch * T, Hq * d, device="cuda", generator=g).to(torch.bfloat16)

    def hide(self, see):
        """NaN at cache rows that no row sees (before packing keeps them out of the 4-bit part's groups: whole rows)."""
        for s, P in enumerate(self.lens):
            dead = torch.from_numpy(~see[s].any(0)).nonzero().flatten().tolist()
            for p in dead:
                page = int(self.eng.page_table[s, p // PAGE])
                if page >= 0:
                    self.eng.kv_pool[:, page, :, :, p % PAGE] = math.nan


def check(out, ref, A, two=False):
    tol = (2.0 ** -15 * ref.abs() + 2.0 ** -11 * A) if two else (2.0 ** -8 * ref.abs() + 2.0 ** -10 * A)
    err = (out.double() - ref).abs()
    assert bool(torch.isfinite(out.double()).all())
    assert bool((err <= tol + 1e-30).all()), float((err / (tol + 1e-30)).max())


def run_attention(cache, kind, window, sinks, seed, two=False, hide=True):
    eng, T = cache.eng, cache.T
    Hq, Hkv, d = cache.heads
    rng = np.random.default_rng(seed)
    batch = len(cache.lens)
    parents = [random_parents(T, rng) for _ in range(batch)] if kind == "tree" else [None] * batch
    see = [visible(P, T, kind, parents[s], window, sinks) for s, P in enumerate(cache.lens)]
    if hide:
        cache.hide(see)
    anc = torch.from_numpy(np.stack([anc_words(p) for p in parents])).cuda() if kind == "tree" else None
    q = cache.q
    q_lo = ((torch.randn(q.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)) * 2.0 ** -9) * q.float().abs()).to(torch.bfloat16) if two else None
    n = batch * T
    guard = torch.full((n + 2, Hq * d), 7.0, dtype=torch.bfloat16, device="cuda")      # rows around the output stay as they are
    out = guard[1 : n + 1]
    lo = torch.zeros_like(q) if two else None
    eng.glance_attention(0, q, T, out, anc=anc, causal=kind == "chain", window=window, sinks=sinks, q_lo=q_lo, out_lo=lo)
    eng.check_device_status()
    assert bool((guard[0] == 7).all()) and bool((guard[-1] == 7).all())
    qd = q.double() + (q_lo.double() if two else 0)
    for s in range(batch):
        ref, A = reference(qd[s * T : (s + 1) * T].view(T, Hq, d), cache.K[s], cache.V[s], see[s])
        got = out[s * T : (s + 1) * T].view(T, Hq, d).double()
        if two:
            got = got + lo[s * T : (s + 1) * T].view(T, Hq, d).double()
        check(got, ref, A, two)
    again = torch.empty_like(out)
    eng.glance_attention(0, q, T, again, anc=anc, causal=kind == "chain", window=window, sinks=sinks, q_lo=q_lo)
    eng.check_device_status()
    if not two:
        assert torch.equal(again, out)                   # the same bits, whatever the timing
    return out


H7, HS, HT = (28, 4, 128), (16, 4, 64), (4, 2, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [H7, HS, HT, (8, 8, 128), (32, 8, 128), (16, 1, 64), (6, 2, 64)])
@pytest.mark.parametrize("layers,lens,tail", [(1, [64], 0), (2, [700, 63, 128, 1000], 0), (3, [130, 500], 65), (1, [0, 1, 64 * 9], 1)])
def test_pack_and_unpack(heads, layers, lens, tail):
    from paper_2609_00355_b200.binding import PackedCache
    eng = make_engine(heads, len(lens), max(lens) + 1, layers)
    g = torch.Generator(device="cuda").manual_seed(5)
    # magnitudes over the format's whole range and beyond: scales that round to 0, subnormal ones, saturated ones
    mag = torch.exp2(torch.randint(-14, 13, eng.kv_pool.shape[:-1] + (eng.kv_pool.shape[-1] // GROUP,), device="cuda", generator=g).float())
    x = (torch.randn(eng.kv_pool.shape, device="cuda", generator=g).unflatten(-1, (-1, GROUP)) * mag[..., None]).flatten(-2).to(torch.bfloat16)
    # ties of the scale and of the codes are common among values of three bits
    x[:, :, :, :, ::2] = (torch.randint(-15, 16, x[:, :, :, :, ::2].shape, device="cuda", generator=g) * 0.25).to(torch.bfloat16)
    eng.kv_pool.copy_(x)
    eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
    packed = PackedCache(eng)
    eng.glance_set_packed(packed)
    eng.glance_pack_cache(keep=tail)
    eng.check_device_status()
    want = [max(0, P - tail) // PAGE * PAGE for P in lens]
    assert packed.len.tolist() == want
    assert torch.equal(eng.kv_pool, x)                   # the bf16 pages are left as they are
    # a part of it back: only pages from there on
    back = torch.full_like(x, 3.0)
    cut = [n // 2 for n in want]
    eng.glance_unpack_cache(torch.tensor(cut, dtype=torch.int32, device="cuda"), kv_pool=back)
    eng.check_device_status()
    assert packed.len.tolist() == [c // PAGE * PAGE for c in cut]
    def pages(a, b):
        return [int(eng.page_table[s, p]) for s in range(len(lens)) for p in range(a[s] // PAGE, b[s] // PAGE)]
    low = [c // PAGE * PAGE for c in cut]
    ref = torch.full(x.shape, 3.0, dtype=torch.float64, device="cuda")
    for p in pages(low, want):
        ref[:, p] = held_values(x[:, p])
    assert torch.equal(back.double(), ref)
    # the rest, and a length beyond what is held changes nothing
    eng.glance_unpack_cache(torch.full((len(lens),), 1 << 30, dtype=torch.int32, device="cuda"), kv_pool=back)
    assert torch.equal(back.double(), ref)
    eng.glance_unpack_cache(torch.zeros(len(lens), dtype=torch.int32, device="cuda"))
    eng.check_device_status()
    assert packed.len.tolist() == [0] * len(lens)
    ref = x.double()
    for p in pages([0] * len(lens), low):
        ref[:, p] = held_values(x[:, p])
    assert torch.equal(eng.kv_pool.double(), ref)


@pytest.mark.gpu
def test_pack_groups_that_are_not_finite_and_signs():
    from paper_2609_00355_b200.binding import PackedCache
    eng = make_engine((4, 2, 64), 1, 128)
    x = torch.randn(eng.kv_pool.shape, device="cuda").to(torch.bfloat16)
    x[..., 3, 5] = math.inf
    x[..., 4, 17] = -math.inf
    x[..., 5, 63] = math.nan
    x[..., 6, :16] = 0.0
    x[..., 7, :16] = 3e38
    x[..., 8, :16] = 1e-38
    eng.kv_pool.copy_(x)
    eng.seq_len.fill_(64)
    eng.glance_set_packed(PackedCache(eng))
    eng.glance_pack_cache()
    eng.glance_unpack_cache(torch.zeros(1, dtype=torch.int32, device="cuda"))
    eng.check_device_status()
    page = int(eng.page_table[0, 0])
    got, ref = eng.kv_pool[:, page].double(), held_values(x[:, page])
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(ref))


CASES = [
    # kind, T, lens, window, sinks
    ("block", 1, [1536], 512, 4), ("block", 1, [0], 1, 0), ("block", 1, [0, 1, 63, 64, 65], 64, 1), ("block", 1, [700, 5, 2000], 1, 0),
    ("block", 1, [2100], 2000, 1), ("block", 1, [3000, 1500], 63, 64), ("block", 1, [900], 65, 129), ("block", 1, [500], 5000, 7),
    ("block", 1, [500], 100, 4000), ("block", 1, [40], 20, 10), ("block", 2, [640], 64, 0), ("block", 4, [333, 1], 130, 3), ("block", 16, [1000], 7, 2),
    ("tree", 2, [128], 1, 0), ("tree", 5, [777, 64], 3, 1), ("tree", 8, [1000], 300, 66), ("tree", 17, [450, 20], 4, 30),
    ("tree", 64, [1536], 700, 4), ("tree", 65, [100, 3000], 64, 64), ("tree", 128, [2048], 1000, 100), ("tree", 128, [5], 6, 8), ("tree", 33, [0], 2, 1),
    ("chain", 3, [70], 2, 1), ("chain", 129, [0], 40, 3), ("chain", 500, [333], 100, 5), ("chain", 300, [64], 1, 0), ("chain", 200, [1000], 1000, 1100),
]


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [H7, HS, (8, 8, 128), (16, 1, 64)])
@pytest.mark.parametrize("kind,T,lens,window,sinks", CASES)
def test_window(heads, kind, T, lens, window, sinks):
    run_attention(Cache(heads, lens, T, 11), kind, window, sinks, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [H7, HS, (8, 8, 128), (16, 1, 64)])
@pytest.mark.parametrize("kind,T,lens,held", [
    ("block", 1, [64], 0), ("block", 1, [1536], 0), ("block", 1, [5000, 300, 64, 0], 64), ("block", 2, [900], 1), ("block", 16, [400, 1500], 130),
    ("tree", 7, [1000], 0), ("tree", 20, [129, 4000], 64), ("tree", 64, [1536], 64), ("tree", 128, [700, 64], 0), ("tree", 100, [20], 0),
    ("chain", 2, [191], 0), ("chain", 400, [512], 0), ("chain", 130, [3000], 500)])
def test_packed(heads, kind, T, lens, held):
    run_attention(Cache(heads, lens, T, 12, held=held), kind, 0, 0, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [H7, HS, HT])
@pytest.mark.parametrize("held", [0, 100, 400])
@pytest.mark.parametrize("kind,T,lens,window,sinks", [
    ("block", 1, [1536, 700], 512, 4), ("block", 1, [1000], 70, 130), ("block", 3, [1000, 100], 200, 64), ("tree", 9, [900], 150, 70),
    ("tree", 64, [1536], 300, 4), ("tree", 80, [2000, 500], 450, 200), ("chain", 300, [900], 333, 65), ("chain", 10, [500], 60, 1)])
def test_packed_window(heads, held, kind, T, lens, window, sinks):
    run_attention(Cache(heads, lens, T, 13, held=held), kind, window, sinks, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [H7, HS])
@pytest.mark.parametrize("held", [None, 64])
@pytest.mark.parametrize("kind,T,lens,window,sinks", [("block", 1, [1536], 512, 4), ("tree", 4, [1000, 300], 300, 4), ("tree", 64, [1536], 700, 4),
                                                      ("chain", 200, [700], 300, 64)])
def test_two_terms(heads, held, kind, T, lens, window, sinks):
    run_attention(Cache(heads, lens, T, 14, held=held), kind, window, sinks, 6, two=True)


@pytest.mark.gpu
def test_zeroed_tiles_side_by_side():
    """The sinks' end and the window's start in neighbouring tiles: rows that nobody sees are cleared in both, and the second may be
    cleared before the first is used."""
    for _ in range(20):
        run_attention(Cache(H7, [2000, 500], 80, 13, held=100), "tree", 450, 200, 5)
        run_attention(Cache(H7, [2000, 500], 80, 13), "tree", 450, 200, 5)


# ---- the target's own passes ---------------------------------------------------------------------------------------
def oracle_pass(sh, tw, K, V, x, pos, P, masks):
    """The target over rows x at cache rows P.. with one visibility mask a layer (the oracle's layer, this file's masks)."""
    from oracle import glance_oracle as O
    rows = torch.arange(P, P + x.shape[0])
    for l, lw in enumerate(tw["layers"]):
        x = O.decoder_layer(sh, lw, x, pos, K[l], V[l], rows, masks[l])
    return O.rmsnorm(x, tw["final_norm"], sh.rms_eps) @ tw["lm_head"].T, x


def seeded_engine(cfg, lens, seed, held=None):
    """An engine and the oracle's widened weights over the same random cache (and what the 4-bit part of it stands for)."""
    from oracle import glance_oracle as O
    from paper_2609_00355_b200.binding import Engine, PackedCache
    tb, hb = synth.make_weights(cfg, "cpu", 0)
    dev = lambda w: {k: ([{a: b.cuda() for a, b in x.items()} for x in v] if isinstance(v, list) else v.cuda()) for k, v in w.items()}
    eng = Engine(cfg, dev(tb), dev(hb), batch=len(lens), max_len=max(lens) + 4 * cfg.tree_N + 256, stream=torch.cuda.Stream())
    with torch.cuda.stream(eng.stream):
        g = torch.Generator(device="cuda").manual_seed(seed)
        eng.kv_pool.copy_(torch.randn(eng.kv_pool.shape, device="cuda", generator=g) * 0.5)
        eng.head_kv_all.copy_(torch.randn(eng.head_kv_all.shape, device="cuda", generator=g) * 0.5)
        eng.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        eng.root.copy_(torch.randint(0, cfg.vocab, (len(lens),), generator=g, device="cuda", dtype=torch.int32))
        cap = max(lens) + 2 * cfg.tree_N + 8
        K = [[torch.zeros(cap, cfg.n_kv_heads, cfg.head_dim) for _ in range(cfg.n_layers)] for _ in lens]
        V = [[torch.zeros(cap, cfg.n_kv_heads, cfg.head_dim) for _ in range(cfg.n_layers)] for _ in lens]
        n4 = [0] * len(lens)
        if held is not None:
            eng.glance_set_packed(PackedCache(eng))
            eng.glance_pack_cache(keep=held)
            n4 = eng.packed.len.tolist()
        for s, P in enumerate(lens):
            for l in range(cfg.n_layers):
                k, v = eng.gather_kv(s, l, P)
                for dst, src in ((K[s][l], k), (V[s][l], v)):
                    dst[:P] = src.float().cpu()
                    dst[: n4[s]] = held_values(src[: n4[s]]).float().cpu()
            for p in range(n4[s] // PAGE):
                eng.kv_pool[:, int(eng.page_table[s, p])] = math.nan
    torch.cuda.synchronize()
    return eng, O.Shape.of(cfg), O.widen(tb), K, V


def relative(got, ref):
    return float((got.double().cpu() - ref.double()).abs().max()) / float(ref.abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("held", [None, 70])
@pytest.mark.parametrize("windows,sinks,N", [((0, 100), 4, 8), ((64, 0), 70, 32), ((30, 300), 0, 1), ((5, 5), 1, 24)])
def test_verify_pass_with_windows_a_layer(windows, sinks, N, held):
    """glance_set_window and glance_set_packed in a verify pass of two layers, ragged batch, against the oracle's layers (logits and
    hidden rows within the 2e-2 of the parity tests); then without them, the same bits as an engine that never had them."""
    from tests import parity_harness as H
    from oracle import glance_oracle as O
    cfg = synth.CONFIGS["tiny"].replace(tree_N=N, batch=2)
    lens = [333, 130]
    eng, sh, tw, K, V = seeded_engine(cfg, lens, 21, held)
    with torch.cuda.stream(eng.stream):
        eng.glance_set_window(windows, sinks)
        rng = np.random.default_rng(4)
        trees = []
        for s, P in enumerate(lens):
            parent = random_parents(N, rng)
            for i in range(1, N):
                parent[i] = max(parent[i], 0)             # one tree, no padding rows
            depth = np.zeros(N, dtype=np.int32)
            for i in range(1, N):
                depth[i] = depth[parent[i]] + 1
            trees.append(O.tree_from_arrays(rng.integers(0, cfg.vocab, N), parent, depth, N))
        H.tree_to_device(eng, trees)
        logits = torch.zeros(2, N, cfg.vocab, device="cuda")
        eng.glance_verify_tree(logits_dbg=logits)
        eng.check_device_status()
        for s, P in enumerate(lens):
            t = trees[s]
            masks = [torch.from_numpy(visible(P, N, "tree", t.parent, w, sinks if w else 0)) for w in windows]
            x = tw["embed"][torch.as_tensor(t.token, dtype=torch.long)].clone()
            ref, hid = oracle_pass(sh, tw, K[s], V[s], x, torch.as_tensor(P + t.depth.astype(np.int64)), P, masks)
            assert relative(logits[s], ref) <= 2e-2
            assert relative(eng.hidden[s], hid) <= 2e-2
    if held is None:
        other, *_ = seeded_engine(cfg, lens, 21)
        with torch.cuda.stream(eng.stream):
            eng.glance_set_window(None)
            eng.kv_pool.copy_(other.kv_pool)
            eng.glance_verify_tree(logits_dbg=logits)
        torch.cuda.synchronize()
        with torch.cuda.stream(other.stream):
            H.tree_to_device(other, trees)
            plain = torch.zeros_like(logits)
            other.glance_verify_tree(logits_dbg=plain)
        torch.cuda.synchronize()
        assert torch.equal(plain, logits)


@pytest.mark.gpu
@pytest.mark.parametrize("prior,count,windows,sinks,held", [(0, 150, (40, 0), 3, None), (200, 77, (64, 100), 65, 0), (333, 130, (0, 50), 0, 100)])
def test_prefill_with_windows(prior, count, windows, sinks, held):
    """A prefill pass of the second sequence of a batch: the new K/V rows of the last layer come from windowed rows of the first."""
    cfg = synth.CONFIGS["tiny"].replace(batch=2)
    eng, sh, tw, K, V = seeded_engine(cfg, [64, prior], 22, held)
    with torch.cuda.stream(eng.stream):
        eng.glance_set_window(windows, sinks)
        emb = torch.randn(count, cfg.hidden, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
        eng.glance_prefill(1, embeds=emb.cuda())
        eng.check_device_status()
        masks = [torch.from_numpy(visible(prior, count, "chain", None, w, sinks if w else 0)) for w in windows]
        oracle_k = [torch.cat([k, torch.zeros(count, *k.shape[1:])]) for k in K[1]]
        oracle_v = [torch.cat([v, torch.zeros(count, *v.shape[1:])]) for v in V[1]]
        oracle_pass(sh, tw, oracle_k, oracle_v, emb.float(), torch.arange(prior, prior + count), prior, masks)
        for l in range(cfg.n_layers):
            k, v = eng.gather_kv(1, l, prior + count)
            assert relative(k[prior:].float(), oracle_k[l][prior : prior + count]) <= 2e-2
            assert relative(v[prior:].float(), oracle_v[l][prior : prior + count]) <= 2e-2
        assert eng.seq_len.tolist() == [64, prior + count]


@pytest.mark.gpu
@pytest.mark.parametrize("name,N", [("tiny", 8), ("tiny", 1), ("small", 32)])
def test_rounds_over_a_packed_cache_replayed_as_a_graph(name, N):
    """Draft, tree, verify, commit and packing as one graph, against the same calls one by one: the same bits, round after round,
    while pages move from bf16 to 4 bits; the cache that is left is what the plain calls leave."""
    from tests import parity_harness as H
    cfg = synth.CONFIGS[name].replace(tree_N=N, batch=2, n_layers=2)
    engs = [seeded_engine(cfg, [190, 127], 23, 64)[0] for _ in range(2)]
    logs = [[], []]
    for which, eng in enumerate(engs):
        with torch.cuda.stream(eng.stream):
            eng.glance_set_window((0, 90), 5)
            logits = torch.zeros(2, N, cfg.vocab, device="cuda")

            def step():
                eng.glance_draft_block()
                eng.glance_build_tree()
                eng.glance_verify_tree(logits_dbg=logits)
                eng.glance_accept_commit()
                eng.glance_pack_cache(keep=64)
            run = step
            if which == 1:
                snap, held = eng.snapshot_state(), eng.packed.len.clone()
                step()
                eng.restore_state(snap)
                eng.packed.len.copy_(held)
                torch.cuda.synchronize()
                run = eng.capture(step).replay
            for _ in range(70):
                run()
                torch.cuda.synchronize()
                logs[which].append((logits.clone(), eng.seq_len.tolist(), eng.packed.len.tolist(), eng.out_tokens.clone()))
            eng.check_device_status()
    for a, b in zip(*logs):
        assert torch.equal(a[0], b[0]) and a[1] == b[1] and a[2] == b[2] and torch.equal(a[3], b[3])
    P, n4 = logs[0][-1][1], logs[0][-1][2]
    assert n4 == [max(0, p - 64) // PAGE * PAGE for p in P] and n4[0] >= 192
    assert torch.equal(engs[0].packed.pool, engs[1].packed.pool)


@pytest.mark.gpu
@pytest.mark.parametrize("taps", [(), (0, 1)])
def test_bf16_pages_of_packed_positions_are_free(taps):
    """With a page table of its own for the block head, rounds do not look at the target's entries of packed pages: the same bits
    with those entries gone and their pages overwritten."""
    from paper_2609_00355_b200.binding import PackedCache
    cfg = synth.CONFIGS["tiny"].replace(tree_N=8, batch=2, head_taps=taps)
    logs = [[], []]
    for which in range(2):
        eng = seeded_engine(cfg, [150, 200], 24)[0]
        with torch.cuda.stream(eng.stream):
            packed = PackedCache(eng, head_page_table=eng.page_table.clone())
            eng.glance_set_packed(packed)
            eng.glance_prefill(0, ids=torch.arange(100, dtype=torch.int32, device="cuda"))
            for _ in range(30):
                eng.glance_pack_cache(keep=10)
                if which == 1:
                    for s, n in enumerate(packed.len.tolist()):
                        for p in range(n // PAGE):
                            if int(eng.page_table[s, p]) >= 0:
                                eng.kv_pool[:, int(eng.page_table[s, p])] = math.nan
                            eng.page_table[s, p] = -1
                eng.round()
                torch.cuda.synchronize()
                logs[which].append((eng.seq_len.tolist(), packed.len.tolist(), eng.out_tokens.clone(), eng.topk_lp.clone(), eng.hidden_all.clone()))
            eng.check_device_status()
            assert packed.len.tolist()[0] >= 192
            head = [eng.gather_head_kv(s, 100) for s in range(2)]
            logs[which].append(head)
    for a, b in zip(logs[0][:-1], logs[1][:-1]):
        assert a[:2] == b[:2] and all(torch.equal(x, y) for x, y in zip(a[2:], b[2:]))
    for a, b in zip(logs[0][-1], logs[1][-1]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.gpu
def test_truncation_into_the_packed_part():
    """Unpack, truncate, go on: the length held falls with the sequence, and stale 4-bit pages are not read."""
    from paper_2609_00355_b200.binding import PackedCache
    cache = Cache(H7, [700, 300], 1, 31)
    eng = cache.eng
    eng.glance_set_packed(PackedCache(eng))
    eng.glance_pack_cache()
    before = eng.kv_pool.clone()
    new_len = torch.tensor([200, 1 << 20], dtype=torch.int32, device="cuda")
    eng.glance_unpack_cache(new_len)
    assert eng.packed.len.tolist() == [192, 256]
    eng.glance_seq_truncate(0, 150, 0)
    eng.check_device_status()
    assert eng.packed.len.tolist() == [128, 256] and eng.seq_len.tolist() == [150, 300]
    assert torch.equal(torch.isnan(eng.kv_pool), torch.isnan(before))
    # new rows from position 150 on, in bf16
    cache.lens = [150, 300]
    for s, P in enumerate(cache.lens):
        K, V = eng.gather_kv(s, 0, P + 1)
        n = eng.packed.len.tolist()[s]
        cache.K[s], cache.V[s] = K.double(), V.double()
        cache.K[s][:n], cache.V[s][:n] = held_values(before_rows(before, eng, s, n)[0]), held_values(before_rows(before, eng, s, n)[1])
    run_attention(cache, "block", 0, 0, 1, hide=False)
    # a sequence that its owner shortened without a word: whole pages beyond it count for nothing
    eng.seq_len.fill_(100)
    cache.lens = [100, 100]
    cache.K = [k[:101] for k in cache.K]
    cache.V = [v[:101] for v in cache.V]
    for s in range(2):
        K, V = eng.gather_kv(s, 0, 101)
        cache.K[s][64:], cache.V[s][64:] = K[64:].double(), V[64:].double()
    run_attention(cache, "block", 0, 0, 1, hide=False)


def before_rows(pool, eng, s, n):
    pos = torch.arange(n, device="cuda")
    pages = eng.page_table[s].long()[pos // PAGE]
    return pool[0][pages, 0, :, pos % PAGE], pool[0][pages, 1, :, pos % PAGE]


# ---- refusals, faults -------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_refusals():
    from paper_2609_00355_b200.binding import GlanceError, PackedCache
    eng = make_engine(HS, 2, 300)
    q = torch.zeros(2 * 200, 16 * 64, dtype=torch.bfloat16, device="cuda")
    anc = torch.ones(2, 4, 1, dtype=torch.int64, device="cuda")

    def refused(what, fn):
        with pytest.raises(GlanceError, match=what):
            fn()
    call = lambda T=4, layer=0, **kw: eng.glance_attention(layer, q[: 2 * T], T, q[: 2 * T].clone(), **kw)
    refused("invalid argument", lambda: call(T=130))                       # a block of more than 128 rows
    refused("invalid argument", lambda: call(layer=1))
    refused("invalid argument", lambda: call(layer=-1))
    refused("invalid argument", lambda: call(window=-1))
    refused("invalid argument", lambda: call(sinks=-1))
    refused("invalid argument", lambda: call(anc=anc, causal=True))
    lib, ref, p = eng.lib, C.byref(eng.seqs), q.data_ptr()
    for args in ((0, None, None, None, 1, 0, 0, 0, p, None), (0, p, None, None, 1, 0, 0, 0, None, None), (0, p + 2, None, None, 1, 0, 0, 0, p, None),
                 (0, p, None, None, 0, 0, 0, 0, p, None), (0, p, None, None, 5000, 1, 0, 0, p, None), (0, p, p + 8, None, 1, 0, 0, 0, p, None)):
        assert lib.glance_attention(eng.ctx, ref, *args) == -1
    assert lib.glance_attention(eng.ctx, None, 0, p, None, None, 1, 0, 0, 0, p, None) == -1
    refused("call order", lambda: eng.glance_pack_cache())
    refused("call order", lambda: eng.glance_unpack_cache(torch.zeros(2, dtype=torch.int32, device="cuda")))
    eng.glance_set_packed(PackedCache(eng))
    refused("invalid argument", lambda: eng.glance_pack_cache(keep=-1))
    assert lib.glance_unpack_cache(eng.ctx, ref, None) == -1
    refused("one window", lambda: eng.glance_set_window([1, 2]))
    refused("invalid argument", lambda: eng.glance_set_window([-1]))
    refused("invalid argument", lambda: eng.glance_set_window([1], -1))
    bad = PackedCache(eng)
    for field in ("len", "page_table", "pool"):
        c = type(bad.c).from_buffer_copy(bad.c)
        setattr(c, field, None)
        assert lib.glance_set_packed(eng.ctx, C.byref(c)) == -1
    c = type(bad.c).from_buffer_copy(bad.c)
    c.pool += 8
    assert lib.glance_set_packed(eng.ctx, C.byref(c)) == -1
    c = type(bad.c).from_buffer_copy(bad.c)
    c.n_pages = 0
    assert lib.glance_set_packed(eng.ctx, C.byref(c)) == -1
    eng.glance_set_packed(None)
    refused("call order", lambda: eng.glance_pack_cache())
    call(T=4, anc=anc)
    eng.check_device_status()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40])
def test_bad_pages_are_reported(T):
    """Page numbers outside a pool are recorded in the status word; nothing outside the pools is read or written."""
    for break_table in ("bf16", "held"):
        cache = Cache(H7, [500], T, 3, held=200)
        eng = cache.eng
        if break_table == "bf16":
            eng.page_table[0, -1] = eng.n_pages
            eng.page_table[0, 500 // PAGE] = -1
        else:
            cache.packed.page_table[0, 2] = cache.packed.n_pages + 5
        out = torch.empty_like(cache.q)
        eng.glance_attention(0, cache.q, T, out)
        assert eng.glance_poll_status() == -6
        # packing pages that are nowhere: reported, the others move
        eng.packed.len.zero_()
        eng.glance_pack_cache(keep=0)
        assert eng.glance_poll_status() == -6


@pytest.mark.gpu
def test_contexts_share_nothing_and_another_stream():
    """Two engines on two streams at once: each has its own workspace."""
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    caches = []
    for k, st in enumerate(streams):
        with torch.cuda.stream(st):
            caches.append(Cache(H7, [3000, 700], 2, 40 + k, held=64, stream=st))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                o = torch.empty_like(caches[k].q)
                caches[k].eng.glance_attention(0, caches[k].q, 2, o, window=1000 * k)
                outs[k].append(o)
    torch.cuda.synchronize()
    for k, st in enumerate(streams):
        with torch.cuda.stream(st):
            want = run_attention(caches[k], "block", 1000 * k, 0, 1, hide=False)
            assert all(torch.equal(want, o) for o in outs[k])


# ---- without a GPU ------------------------------------------------------------------------------------------------------
def test_host_arguments_and_sizes():
    from paper_2609_00355_b200 import binding
    from paper_2609_00355_b200 import build as glance_build
    glance_build.build()
    lib = binding.load_library()
    assert lib.glance_set_window(None, None, 0) == -1
    assert lib.glance_set_packed(None, None) == -1
    assert lib.glance_pack_cache(None, None, 0) == -1
    assert lib.glance_unpack_cache(None, None, None) == -1
    assert lib.glance_attention(None, None, 0, None, None, None, 1, 0, 0, 0, None, None) == -1
    for name, d in (("7b", 128), ("small", 64)):
        cfg = synth.CONFIGS[name]
        cc = binding.make_config(cfg, 1, 100)
        assert lib.glance_packed_bytes(C.byref(cc), 7) == cfg.n_layers * 7 * cfg.n_kv_heads * 2 * 64 * (d // 2 + d // 16)
        assert lib.glance_packed_bytes(C.byref(cc), 0) == 0
    assert lib.glance_packed_bytes(None, 3) == 0
    cc.page_size = 32
    assert lib.glance_packed_bytes(C.byref(cc), 7) == 0


def test_definition_of_the_four_bit_values():
    """The reference of these tests on values whose result is plain: ties, saturation, zeros, groups that are not finite."""
    x = torch.zeros(8, 16)
    x[0] = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, 0.26, 0.24, 4.9, 5.1, 0.0])      # scale 1
    x[1, 0] = 6 * 17 / 16                                # scale between 1 and 1.125: the even code, 1
    x[2, 0] = 1e9                                        # scale 448
    x[3, 0] = 2.0 ** -10                                 # scale below half the smallest
    x[4, :2] = torch.tensor([math.inf, 1.0])
    x[5, :2] = torch.tensor([math.nan, 1.0])
    v = held_values(x)
    assert v[0].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.0, -1.0, -4.0, 0.5, 0.0, 4.0, 6.0, 0.0]
    assert float(v[1, 0]) == 6.0 and float(v[2, 0]) == 2688.0 and float(v[3].abs().max()) == 0.0
    assert bool(torch.isnan(v[4]).all()) and bool(torch.isnan(v[5]).all())
    assert torch.equal(v[:4].float().to(torch.bfloat16).double(), v[:4])                                    # exact in bf16


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kind,T,lens,window,sinks,held", [
    (H7, "tree", 4, [7000], 0, 0, 64), (H7, "tree", 5, [20000], 19000, 100, None), (HS, "tree", 8, [9000], 0, 0, 5000), (H7, "tree", 18, [6500], 6300, 0, 64),
    ((16, 1, 64), "block", 3, [30000], 0, 0, 0), (H7, "tree", 4, [100], 0, 0, 0), ((8, 8, 128), "tree", 30, [7000], 0, 0, 3000),
    (H7, "chain", 20, [9000], 8500, 7, 300), (HT, "block", 16, [40000], 0, 0, 64)])
def test_tiles_split_over_several_clusters(heads, kind, T, lens, window, sinks, held):
    """Few tiles over a long table: every tile's clusters meet in global memory.  Also where the sequence is much shorter than the
    table, so that most clusters have nothing."""
    cache = Cache(heads, lens + ([] if lens[0] > 5000 else [7000]), T, 51, held=held)
    run_attention(cache, kind, window, sinks, 8)
    run_attention(cache, kind, window, sinks, 9, two=True, hide=False)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,lens,window,sinks,held", [
    (H7, [33000], 0, 0, 64), (H7, [5000 + 37 * i for i in range(16)], 0, 0, 100), (H7, [1, 0, 9000, 64, 63, 128], 4000, 70, 64), (HS, list(range(64)), 20, 2, 0),
    (H7, [40 * i for i in range(16)], 0, 0, None), (H7, [40 * i for i in range(16)], 0, 0, 64), (HS, [37 * i for i in range(7)], 100, 3, 64),
    ((32, 8, 128), [3000 - 41 * i for i in range(20)], 0, 0, None), ((8, 8, 128), [12000, 1], 11000, 0, None), ((16, 1, 64), [50, 20000, 7], 0, 0, 3000)])
def test_stretches_of_a_batch(heads, lens, window, sinks, held):
    """Single tokens of ragged batches: stretches that begin and end inside an item, items shared by many CTAs, even shares."""
    cache = Cache(heads, lens, 1, 52, held=held)
    run_attention(cache, "block", window, sinks, 8)
    run_attention(cache, "block", window, sinks, 9, two=True, hide=False)


@pytest.mark.gpu
@pytest.mark.parametrize("held", [None, 64])
@pytest.mark.parametrize("heads,n", [(H7, 23), ((32, 8, 128), 13), ((16, 1, 64), 61)])
def test_stretches_that_end_between_items(heads, n, held):
    """Many items of very different lengths: a CTA takes short ones whole, and stretches begin and end before an item's first page."""
    cache = Cache(heads, [(i * i * 131) % 4001 for i in range(n)], 1, 53, held=held)
    run_attention(cache, "block", 0, 0, 8)
    run_attention(cache, "block", 0, 0, 9, two=True, hide=False)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,T", [(H7, 2), (H7, 40), (HS, 3), (HS, 70)])
def test_rows_that_see_nothing_are_zeros(heads, T):
    """Empty sets over no context, in one call with rows that see something; and sets without the row itself."""
    Hq, Hkv, d = heads
    cache = Cache(heads, [0, 300], T, 61)
    eng = cache.eng
    W = (T + 63) // 64
    anc = torch.zeros(2, T, W, dtype=torch.int64, device="cuda")
    anc[0, 1, 0] = 1                                     # sequence 0: only row 1 sees anything: row 0
    anc[1, :, 0] = 2                                     # sequence 1: everybody sees row 1 and a window of the context
    out = torch.full_like(cache.q, 9.0)
    eng.glance_attention(0, cache.q, T, out, anc=anc, window=50)
    eng.check_device_status()
    out = out.view(2, T, Hq, d)
    assert float(out[0, [i for i in range(T) if i != 1]].abs().max()) == 0.0
    assert torch.equal(out[0, 1].view(Hkv, -1, d).double(), cache.V[0][0][:, None].expand(-1, Hq // Hkv, -1))
    see = np.zeros((T, 300 + T), dtype=bool)
    see[:, 301] = True
    see[:, 300 - 49 : 300] = True                        # a set of one stands at the first position
    ref, A = reference(cache.q.view(2, T, Hq, d)[1].double(), cache.K[1], cache.V[1], see)
    check(out[1], ref, A)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 30])
def test_pools_beyond_four_gigabytes(T):
    """Pages whose bytes lie beyond 2^32 in the bf16 pool of a layer and in the 4-bit pool."""
    from paper_2609_00355_b200.binding import PackedCache
    heads, P = H7, 1000
    cache = Cache(heads, [P], T, 71)
    big = make_engine(heads, 1, 40000 * PAGE)
    assert big.kv_pool.numel() * 2 > 1 << 32
    n = (P + T + PAGE - 1) // PAGE
    pages = torch.arange(big.n_pages - n, big.n_pages, dtype=torch.int32, device="cuda")
    big.page_table[0, :n] = pages
    for p in range(n):
        big.kv_pool[:, int(pages[p])] = cache.eng.kv_pool[:, int(cache.eng.page_table[0, p])]
    big.seq_len.fill_(P)
    packed = PackedCache(big, n_pages=130000)
    assert packed.pool.numel() > 1 << 32
    packed.page_table[0, :n] = torch.arange(130000 - n, 130000, dtype=torch.int32, device="cuda")
    big.glance_set_packed(packed)
    small, cache.eng = cache.eng, big
    run_attention(cache, "tree", 700, 30, 2, hide=False)
    big.glance_pack_cache(keep=100)
    held = int(packed.len[0])
    assert held == 896
    cache.K[0][:held], cache.V[0][:held] = held_values(cache.K[0][:held]), held_values(cache.V[0][:held])
    big.kv_pool[:, pages[: held // PAGE].long()] = math.nan
    run_attention(cache, "tree", 0, 0, 2, hide=False)
    big.glance_unpack_cache(torch.zeros(1, dtype=torch.int32, device="cuda"))
    run_attention(cache, "tree", 0, 0, 2, hide=False)


@pytest.mark.gpu
def test_a_snapshot_takes_the_length_held_in_four_bits_along():
    """Back to a snapshot, other rows from there on: pages packed in between are not read."""
    cfg = synth.CONFIGS["tiny"].replace(tree_N=8, batch=1)
    logs = [[], []]
    for which in range(2):
        eng = seeded_engine(cfg, [180], 25, 50)[0]
        with torch.cuda.stream(eng.stream):
            snap = eng.snapshot_state()
            assert len(snap) == 5
            if which == 1:
                eng.root.fill_(7)
                for _ in range(30):
                    eng.round()
                eng.glance_pack_cache()
                assert eng.packed.len.tolist()[0] >= 192
                eng.restore_state(snap)
                assert eng.packed.len.tolist() == [128]
            for _ in range(20):
                eng.round()
                torch.cuda.synchronize()
                logs[which].append((eng.seq_len.clone(), eng.out_tokens.clone(), eng.hidden_all.clone()))
            eng.check_device_status()
    for a, b in zip(*logs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_snapshot_from_before_the_pool_bounds_the_length_held():
    """restore_state on host tensors: whole pages of the restored length are the most that stays held in 4 bits."""
    from types import SimpleNamespace

    from paper_2609_00355_b200.binding import Engine
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    eng = SimpleNamespace(cfg=SimpleNamespace(page_size=PAGE), seq_len=i32(180, 700, 63, 640), root=i32(1, 2, 3, 4),
                          feat_all=torch.zeros(1, 4, 2, 8), feat_count=i32(0, 0, 0, 0))
    snap = Engine.snapshot_state(eng)
    assert len(snap) == 4
    eng.packed = SimpleNamespace(len=i32(256, 640, 64, 640))
    later = Engine.snapshot_state(eng)
    eng.seq_len.add_(200)
    Engine.restore_state(eng, snap)
    assert eng.seq_len.tolist() == [180, 700, 63, 640]
    assert eng.packed.len.tolist() == [128, 640, 0, 640]
    eng.packed.len.copy_(i32(320, 832, 128, 768))
    Engine.restore_state(eng, later)
    assert eng.packed.len.tolist() == [128, 640, 0, 640]


@pytest.mark.gpu
def test_back_to_a_snapshot_from_before_the_pool():
    """Snapshot, register a pool, run and pack, go back, run on: rows written since are not read from 4-bit pages.  The same
    bits as an engine that packed at the snapshot's length."""
    from paper_2609_00355_b200.binding import PackedCache
    cfg = synth.CONFIGS["tiny"].replace(tree_N=8, batch=1)
    logs = [[], []]
    for which in range(2):
        eng = seeded_engine(cfg, [180], 25)[0]
        with torch.cuda.stream(eng.stream):
            snap = eng.snapshot_state()
            eng.glance_set_packed(PackedCache(eng))
            if which == 1:
                eng.root.fill_(7)
                for _ in range(30):
                    eng.round()
                eng.glance_pack_cache()
                assert eng.packed.len.tolist()[0] >= 192
                eng.restore_state(snap)
            else:
                eng.glance_pack_cache()
            assert eng.packed.len.tolist() == [128]
            for _ in range(30):
                eng.round()
                torch.cuda.synchronize()
                logs[which].append((eng.seq_len.clone(), eng.out_tokens.clone(), eng.hidden_all.clone()))
            eng.check_device_status()
    for a, b in zip(*logs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.gpu
@pytest.mark.parametrize("heads,layers", [(H7, 2), (HS, 3)])
def test_packing_stops_before_a_page_without_a_place(heads, layers):
    """A pool with fewer pages than the sequences: the lengths rise as far as there are places, pages that have one move, the
    call reports it, and attention over what is there is right; with the places given, the rest follows."""
    from paper_2609_00355_b200.binding import PackedCache
    lens, T = [700, 300, 130, 1000], 2
    cache = Cache(heads, lens, T, 91, layers=layers)
    eng, x = cache.eng, cache.eng.kv_pool.clone()
    packed = PackedCache(eng)
    table, own = eng.page_table.clone(), packed.page_table.clone()
    packed.page_table[0, 6] = -1                         # sequence 0 ends in the pool after six pages
    packed.page_table[0, 8] = packed.n_pages
    packed.page_table[1, 4] = -5                         # not due: 300 positions are four pages
    packed.page_table[3, 0] = packed.n_pages + 3         # sequence 3 finds none at all
    eng.page_table[2, 1] = eng.n_pages                   # and a page that is not in the bf16 pool cannot move either
    eng.glance_set_packed(packed)
    eng.glance_pack_cache()
    assert eng.glance_poll_status() == -6
    assert packed.len.tolist() == [6 * 64, 4 * 64, 64, 0]
    assert torch.equal(torch.nan_to_num(eng.kv_pool), torch.nan_to_num(x))
    eng.glance_pack_cache()                              # it stays so
    assert eng.glance_poll_status() == -6
    assert packed.len.tolist() == [6 * 64, 4 * 64, 64, 0]
    eng.page_table.copy_(table)
    K, V = [k.clone() for k in cache.K], [v.clone() for v in cache.V]

    def compare():
        for s, n in enumerate(packed.len.tolist()):
            cache.K[s], cache.V[s] = K[s].clone(), V[s].clone()
            cache.K[s][:n], cache.V[s][:n] = held_values(K[s][:n]), held_values(V[s][:n])
        run_attention(cache, "block", 0, 0, 1, hide=False)
        run_attention(cache, "block", 200, 70, 1, hide=False)
    compare()
    packed.page_table.copy_(own)
    eng.glance_pack_cache()
    eng.check_device_status()
    assert packed.len.tolist() == [P // 64 * 64 for P in lens]
    compare()


@pytest.mark.gpu
@pytest.mark.parametrize("heads,layers", [(H7, 2), (HS, 3)])
def test_unpacking_stops_behind_a_page_without_a_place(heads, layers):
    """The way back: a length does not fall below a page that could not be written; the others due are written, no more."""
    from paper_2609_00355_b200.binding import PackedCache
    lens, T = [700, 300, 130, 1000], 2
    cache = Cache(heads, lens, T, 92, layers=layers)
    eng, x = cache.eng, cache.eng.kv_pool.clone()
    packed = PackedCache(eng)
    eng.glance_set_packed(packed)
    eng.glance_pack_cache()
    eng.check_device_status()
    K, V = [k.clone() for k in cache.K], [v.clone() for v in cache.V]
    table, own = eng.page_table.clone(), packed.page_table.clone()
    eng.page_table[0, 2] = -1                            # due from page 1 on: pages 6.. are back
    eng.page_table[0, 5] = eng.n_pages
    eng.page_table[1, 0] = -1                            # not due
    packed.page_table[3, 14] = -1                        # the last one held has no place to be read from: nothing is back
    back = torch.full_like(x, 3.0)
    eng.glance_unpack_cache(torch.tensor([64, 128, 1 << 20, 0], dtype=torch.int32, device="cuda"), kv_pool=back)
    assert eng.glance_poll_status() == -6
    assert packed.len.tolist() == [6 * 64, 128, 128, 15 * 64]
    ref = torch.full(x.shape, 3.0, dtype=torch.float64, device="cuda")
    for s, pages in ((0, (1, 3, 4, 6, 7, 8, 9)), (1, (2, 3)), (3, range(14))):
        for p in pages:
            ref[:, int(table[s, p])] = held_values(x[:, int(table[s, p])])
    assert torch.equal(back.double(), ref)
    packed.page_table.copy_(own)
    for s, n in enumerate(packed.len.tolist()):
        cache.K[s][:n], cache.V[s][:n] = held_values(K[s][:n]), held_values(V[s][:n])
    eng.page_table[0, :6] = -1                           # what is held is read from where it is held
    run_attention(cache, "block", 0, 0, 1, hide=False)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [H7, HS])
@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("kind,T,lens,window,sinks,held", [
    ("block", 1, [1536], 512, 4, None), ("block", 1, [1536], 512, 4, 64), ("block", 1, [40, 64, 700], 100, 0, 64), ("block", 2, [0, 300], 0, 0, 64),
    ("block", 1, [9000], 0, 0, 64), ("block", 1, [500, 6000, 100], 0, 0, 64), ("tree", 64, [1536], 512, 4, None), ("tree", 40, [700, 64], 0, 0, 64),
    ("tree", 8, [9000], 0, 0, 64), ("chain", 200, [300], 100, 5, None)])
def test_a_nan_in_a_query_stays_in_its_row(heads, two, kind, T, lens, window, sinks, held):
    """Whatever plan a launch has: every output of a query with a NaN is NaN, and the other rows keep their bits."""
    cache = Cache(heads, lens, T, 81, held=held)
    eng, (Hq, Hkv, d) = cache.eng, heads
    rng = np.random.default_rng(1)
    anc = torch.from_numpy(np.stack([anc_words(np.arange(T) - 1) for _ in lens])).cuda() if kind == "tree" else None
    n = len(lens) * T
    call = lambda q, q_lo, out, lo: eng.glance_attention(0, q, T, out, anc=anc, causal=kind == "chain", window=window, sinks=sinks, q_lo=q_lo, out_lo=lo)
    lo_in = (cache.q * 2.0 ** -9).contiguous() if two else None
    outs = []
    bad = sorted({(int(rng.integers(0, n)), int(rng.integers(0, Hq))) for _ in range(3)})
    q = cache.q.clone()
    for r, h in bad:
        q[r, h * d + int(rng.integers(0, d))] = math.nan
    for x in (cache.q, q):
        out = torch.zeros_like(x)
        lo = torch.zeros_like(x) if two else None
        call(x, lo_in, out, lo)
        eng.check_device_status()
        outs.append([o.view(n, Hq, d) for o in (out, lo) if o is not None])
    for clean, got in zip(*outs):
        assert bool(torch.isfinite(clean).all())
        for r, h in bad:
            assert bool(torch.isnan(got[r, h]).all())
            got[r, h] = clean[r, h]
        assert torch.equal(got, clean)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [H7, (8, 8, 128), HT])
@pytest.mark.parametrize("kind,T,window,held", [("block", 1, 0, None), ("block", 1, 0, 64), ("block", 1, 500, 64), ("tree", 2, 0, 64), ("tree", 40, 0, None),
                                                ("tree", 40, 300, 64), ("chain", 200, 0, 64), ("chain", 200, 100, None)])
def test_lengths_beyond_the_page_table_are_reported(heads, kind, T, window, held):
    """Up to the largest 32-bit length, where positions and page counts would pass 32 bits: the status word says so, and the
    other sequences' rows are right."""
    lens = [300, 2000, 40, 1500, 64]
    cache = Cache(heads, lens, T, 96, held=held)
    eng, (Hq, Hkv, d) = cache.eng, heads
    cap = eng.pages_per_seq * PAGE
    anc = torch.from_numpy(np.stack([anc_words(np.arange(T) - 1) for _ in lens])).cuda() if kind == "tree" else None
    out = torch.empty_like(cache.q)
    call = lambda: eng.glance_attention(0, cache.q, T, out, anc=anc, causal=kind == "chain", window=window, sinks=3)
    for long in ((2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1 - T, 2 ** 31 - 64), (1 << 30, cap), (cap - T + 1, cap - T + 1)):
        eng.seq_len[1], eng.seq_len[3] = long
        call()
        assert eng.glance_poll_status() == -6
        for s in (0, 2, 4):
            see = visible(lens[s], T, kind, np.arange(T) - 1, window, 3)
            ref, A = reference(cache.q.view(-1, T, Hq, d)[s].double(), cache.K[s], cache.V[s], see)
            check(out.view(-1, T, Hq, d)[s], ref, A)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [H7, HS])
@pytest.mark.parametrize("two", [False, True])
@pytest.mark.parametrize("kind,T,lens,window,sinks,held", [
    ("block", 1, [1536], 512, 4, None), ("block", 1, [1536], 512, 4, 64), ("block", 1, [0, 64, 700], 1, 0, 64), ("block", 2, [0, 300], 0, 0, 64),
    ("block", 1, [9000], 0, 0, 64), ("block", 1, [500, 6000, 100], 0, 0, 64), ("tree", 64, [1536], 512, 4, None), ("tree", 40, [700, 64], 0, 0, 64),
    ("tree", 8, [9000], 0, 0, 64), ("chain", 200, [300], 100, 5, None), ("chain", 1300, [70], 0, 0, 0)])
def test_an_infinite_query_gives_nan(heads, two, kind, T, lens, window, sinks, held):
    """All its scores are -inf where its sign differs from every key's: 0 / 0 by the definition, not a row that sees nothing."""
    cache = Cache(heads, lens, T, 82)
    eng, (Hq, Hkv, d) = cache.eng, heads
    eng.kv_pool[:, :, 0, :, :, 3] = -1 - eng.kv_pool[:, :, 0, :, :, 3].abs()
    if held is not None:
        from paper_2609_00355_b200.binding import PackedCache
        eng.glance_set_packed(PackedCache(eng))
        eng.glance_pack_cache(keep=held)
    rng = np.random.default_rng(2)
    anc = torch.from_numpy(np.stack([anc_words(np.arange(T) - 1) for _ in lens])).cuda() if kind == "tree" else None
    n = len(lens) * T
    bad = sorted({(int(rng.integers(0, n)), int(rng.integers(0, Hq))): (-1) ** i for i in range(4)}.items())
    q = cache.q.clone()
    for (r, h), sign in bad:
        q[r, h * d + 3] = sign * math.inf
    outs = []
    for x in (cache.q, q):
        out = torch.zeros_like(x)
        lo = torch.zeros_like(x) if two else None
        eng.glance_attention(0, x, T, out, anc=anc, causal=kind == "chain", window=window, sinks=sinks,
                             q_lo=(cache.q * 2.0 ** -9).contiguous() if two else None, out_lo=lo)
        eng.check_device_status()
        outs.append([o.view(n, Hq, d) for o in (out, lo) if o is not None])
    for clean, got in zip(*outs):
        assert bool(torch.isfinite(clean).all())
        for (r, h), _ in bad:
            assert bool(torch.isnan(got[r, h]).all())
            got[r, h] = clean[r, h]
        assert torch.equal(got, clean)


def test_tensors_of_another_device_are_refused():
    """A pointer into another GPU's memory would fault on this one: refused before the library is called."""
    from types import SimpleNamespace

    from paper_2609_00355_b200.binding import Engine, PackedCache

    def tensor(dtype, n, index=0):
        return SimpleNamespace(dtype=dtype, numel=lambda: n, shape=(1, n), get_device=lambda: index, is_cuda=True, is_contiguous=lambda: True,
                               data_ptr=lambda: 1 << 20)
    called = []
    eng = SimpleNamespace(batch=1, device_index=0, ctx=None, seqs=C.c_int(), ccfg=SimpleNamespace(n_q_heads=4, head_dim=64),
                          kv_pool=tensor(torch.bfloat16, 8),
                          lib=SimpleNamespace(glance_attention=lambda *a: called.append(a) or 0, glance_unpack_cache=lambda *a: called.append(a) or 0))
    row = lambda index=0: tensor(torch.bfloat16, 256, index)
    Engine.glance_attention(eng, 0, row(), 1, row(), anc=tensor(torch.int64, 1), q_lo=row(), out_lo=row())
    Engine.glance_unpack_cache(eng, tensor(torch.int32, 1))
    assert len(called) == 2
    for args, kw in (((row(1), row()), {}), ((row(), row(1)), {}), ((row(), row()), dict(anc=tensor(torch.int64, 1, 1))),
                     ((row(), row()), dict(q_lo=row(1))), ((row(), row()), dict(out_lo=row(1)))):
        with pytest.raises(AssertionError, match="the engine's device"):
            Engine.glance_attention(eng, 0, args[0], 1, args[1], **kw)
    with pytest.raises(AssertionError, match="the engine's device"):
        Engine.glance_unpack_cache(eng, tensor(torch.int32, 1, 1))
    with pytest.raises(AssertionError, match="the engine's device"):
        Engine.glance_unpack_cache(eng, tensor(torch.int32, 1), kv_pool=tensor(torch.bfloat16, 8, 1))
    eng.page_table = tensor(torch.int32, 3)
    with pytest.raises(AssertionError, match="the engine's device"):
        PackedCache(eng, head_page_table=tensor(torch.int32, 3, 1))
    assert len(called) == 2


def test_a_pool_made_for_another_engine_is_refused():
    """Its page table or its pages have another size, or it lies on another device: the kernels would read beyond it."""
    from types import SimpleNamespace

    from paper_2609_00355_b200 import binding
    from paper_2609_00355_b200 import build as glance_build
    glance_build.build()
    lib = binding.load_library()
    called = []

    def engine(name, pages):
        return SimpleNamespace(ccfg=binding.make_config(synth.CONFIGS[name], 2, pages), page_table=torch.zeros(2, pages), device_index=0, ctx=None,
                               lib=SimpleNamespace(glance_packed_bytes=lib.glance_packed_bytes, glance_set_packed=lambda *a: called.append(a) or 0))

    def packed(eng, n_pages, index=0):
        nbytes = lib.glance_packed_bytes(C.byref(eng.ccfg), n_pages)
        return SimpleNamespace(n_pages=n_pages, page_table=eng.page_table, pool=SimpleNamespace(numel=lambda: nbytes, get_device=lambda: index), c=binding.Packed())
    small, longer, wide = engine("small", 9), engine("small", 10), engine("7b", 9)
    fits = packed(small, 5)
    binding.Engine.glance_set_packed(small, fits)
    assert small.packed is fits and len(called) == 1
    for other in (packed(longer, 5), packed(wide, 5), packed(small, 5, index=1)):
        with pytest.raises(binding.GlanceError, match="another engine"):
            binding.Engine.glance_set_packed(small, other)
    assert small.packed is fits and len(called) == 1
    binding.Engine.glance_set_packed(small, None)
    assert small.packed is None and len(called) == 2
