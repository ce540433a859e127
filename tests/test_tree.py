"""Attention of drafted tokens over the paged cache: refusals (CPU) and outputs
against the fp64 loops of the definition (GPU).

Tolerance, element by element: 2^-8 of |ref| for the bf16 output, 2^-8 of every
|weight * value| for the weights' rounding to bf16, and what d + 8 roundings of
2^-24 in a score can change (`slack` of serve_ref.tree)."""
import ctypes
import threading

import numpy as np
import pytest
import torch

from paper_2402_17152_amd import hstu
from tests import serve_ref as ref

P = ctypes.c_void_p
FAKE = 0x10000
KINDS = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _problem(**kw):
    a = dict(num_seqs=2, total_tokens=10, max_seq_len=100, num_heads=2, d_qk=64, d_v=32,
             num_time_buckets=8, dtype=hstu.HSTU_BF16)
    a.update(kw)
    return hstu.make_problem(**a)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(p=dict(dtype=hstu.HSTU_F32)), 2, "bf16"), (dict(p=dict(num_heads=65)), 2, "num_heads"),
    (dict(c=None), 1, "cache is NULL"), (dict(c=dict(lengths=None)), 1, "lengths"),
    (dict(c=dict(page_size=24)), 2, "page_size"), (dict(j=None), 1, "jagged"),
    (dict(j=dict(rab_time=None)), 1, "rab_time"), (dict(draft=0), 1, "max_draft"),
    (dict(draft=1025), 2, "max_draft"), (dict(draft=4), 1, "10 drafted"), (dict(q=None), 1, "q is"),
    (dict(ks=64), 1, "k_stride"), (dict(v=FAKE + 8), 1, "v is not"), (dict(out=None), 1, "out"),
    (dict(ws=None), 3, "NULL"), (dict(ws=FAKE + 16), 3, "aligned"), (dict(wsb=16), 3, "too small"),
])
def test_refusals(kw, status, needle):
    p = _problem(**kw.get("p", {}))
    c = dict(num_pages=8, page_size=64, max_pages=4, dtype=hstu.HSTU_CACHE_E4M3, k=FAKE, v=FAKE,
             k_scale=FAKE, v_scale=FAKE, timestamps=FAKE, page_table=FAKE, lengths=FAKE)
    c = None if kw.get("c", 0) is None else hstu.CacheDesc(**{**c, **kw.get("c", {})})
    j = dict(seq_offsets=FAKE, timestamps=FAKE, num_targets=None, rab_pos=FAKE, rab_time=FAKE)
    j = None if kw.get("j", 0) is None else hstu.Jagged(**{**j, **kw.get("j", {})})
    g = lambda n, d: kw.get(n, d)  # noqa: E731
    st = hstu.lib.hstu_attn_fwd_tree(
        ctypes.byref(p), None if j is None else ctypes.byref(j),
        None if c is None else ctypes.byref(c), None, g("draft", 16), P(g("q", FAKE)),
        g("qs", 128), P(g("k", FAKE)), g("ks", 128), P(g("v", FAKE)), g("vs", 64),
        P(g("out", FAKE)), P(g("ws", FAKE)), g("wsb", 1 << 40), None)
    assert st == status
    assert needle in hstu.hstu_last_error()


def test_workspace_and_positions_refusals():
    def desc(**kw):
        return hstu.CacheDesc(**{**dict(num_pages=8, page_size=64, max_pages=4,
                                        dtype=hstu.HSTU_CACHE_INT8), **kw})

    def need(p, c, n):
        return hstu.lib.hstu_attn_fwd_tree_workspace_bytes(ctypes.byref(p), ctypes.byref(c), n)
    n = need(_problem(), desc(), 16)
    assert n > 0 and n % 256 == 0
    assert need(_problem(), desc(page_size=5), 16) == 0
    assert need(_problem(d_v=16), desc(), 16) == 0
    assert need(_problem(), desc(), 0) == 0 and need(_problem(), desc(), 1025) == 0

    def positions(B=2, T=10, n=8, offs=FAKE, out=FAKE):
        return hstu.lib.hstu_tree_positions(B, T, n, P(offs), None, None, P(out), None)
    for st, status in ((positions(B=0), 1), (positions(T=-1), 1), (positions(n=0), 1),
                       (positions(n=2000), 2), (positions(offs=None), 1),
                       (positions(out=None), 1), (positions(T=0, out=None), 0)):
        assert st == status


def test_more_workgroups_than_a_launch_has():
    c = hstu.CacheDesc(num_pages=8, page_size=256, max_pages=1, dtype=hstu.HSTU_CACHE_INT8)
    p = _problem(num_seqs=(1 << 24) // 16, num_heads=64)
    assert hstu.lib.hstu_attn_fwd_tree_workspace_bytes(ctypes.byref(p), ctypes.byref(c), 1) == 0
    assert "sequences of 1 drafted" in hstu.hstu_last_error()
    p = _problem(num_seqs=1 << 20, num_heads=1)
    assert hstu.lib.hstu_attn_fwd_tree_workspace_bytes(ctypes.byref(p), ctypes.byref(c), 64) == 0
    st = hstu.lib.hstu_tree_positions(1 << 24, 10, 8, P(FAKE), None, None, P(FAKE), None)
    assert st == 2 and "sequences" in hstu.hstu_last_error()


def test_binding_refusals(monkeypatch):
    monkeypatch.setattr(hstu, "_raw_device", lambda: 0)
    cache = hstu.PagedCache(torch.zeros(4, 2, 16, 32).bfloat16(),
                            torch.zeros(4, 2, 64, 16).bfloat16(),
                            torch.zeros(4, 16, dtype=torch.int64),
                            torch.zeros(3, 2, dtype=torch.int32),
                            torch.zeros(3, dtype=torch.int64))
    q, v = torch.zeros(6, 2, 32).bfloat16(), torch.zeros(6, 2, 64).bfloat16()
    base = dict(q=q, k=q, v=v, seq_offsets=torch.tensor([0, 2, 4, 6]),
                timestamps=torch.arange(6), cache=cache, rab_pos=torch.zeros(39),
                rab_time=torch.zeros(8), max_seq_len=20, max_draft=2)
    for kw, err, needle in [
            (dict(seq_offsets=torch.tensor([0, 6])), ValueError, "a cache of 3"),
            (dict(seq_offsets=torch.tensor([0, 2, 4, 6]).int()), TypeError, "seq_offsets"),
            (dict(k=q.float()), TypeError, "k must be"), (dict(v=q), ValueError, "v must be"),
            (dict(q=q[:, :1], k=q[:, :1]), ValueError, "q must be"),
            (dict(timestamps=torch.arange(5)), ValueError, "timestamps"),
            (dict(parents=torch.zeros(6).int()), TypeError, "parents"),
            (dict(parents=torch.zeros(7).long()), ValueError, "parents"),
            (dict(rab_pos=torch.zeros(40)), ValueError, "rab_pos"),
            (dict(rab_time=torch.zeros(8).double()), TypeError, "rab_time"),
            (dict(out=torch.zeros(6, 2, 32).bfloat16()), ValueError, "out must be"),
            (dict(max_draft=0), ValueError, "current device"),
            (dict(), ValueError, "current device")]:
        with pytest.raises(err, match=needle):
            hstu.hstu_attn_fwd_tree(**{**base, **kw})


# ------------------------------------------------------------------- GPU

class Batch:
    """Users with cached tokens (on random pages) and drafted ones, the cache
    filled by hstu_cache_write."""

    def __init__(self, hist, nodes, h=2, dqk=64, dv=64, kind="e4m3", page=32, shape="tree", N=None,
                 seed=0, scale=1.0, nb=64):
        g = torch.Generator().manual_seed(seed)
        r = np.random.default_rng(seed)
        self.hist, self.nodes, self.kind, self.h, self.dqk, self.dv = hist, nodes, kind, h, dqk, dv
        B, M, T = len(hist), sum(hist), sum(nodes)
        self.B, self.T = B, T
        self.N = N or max([a + b for a, b in zip(hist, nodes)] + [1])
        if shape == "chain":
            par = [list(range(-1, n - 1)) for n in nodes]
        elif shape == "flat":
            par = [[-1] * n for n in nodes]
        elif shape == "comb":  # deep, with leaves hanging off the spine
            par = [[max(-1, i - 2) if i % 3 == 0 else i - 1 for i in range(n)] for n in nodes]
        else:
            par = [[int(r.integers(max(-1, i - 9), i)) for i in range(n)] for n in nodes]
        self.par = par
        z = torch.randn(T, 2 * h * (dqk + dv), generator=g).mul(scale).bfloat16().cuda()
        c = [h * dv, 2 * h * dv, 2 * h * dv + h * dqk]
        self.v = z[:, c[0]:c[1]].unflatten(1, (h, dv))
        self.q = z[:, c[1]:c[2]].unflatten(1, (h, dqk))
        self.k = z[:, c[2]:].unflatten(1, (h, dqk))
        self.kc = torch.randn(M, h, dqk, generator=g).mul(scale).bfloat16()
        self.vc = torch.randn(M, h, dv, generator=g).mul(scale).bfloat16()
        self.tc = torch.randint(0, 1 << 34, (M,), generator=g)
        self.t = torch.randint(0, 1 << 34, (T,), generator=g)
        self.rab_pos = 0.3 * torch.randn(2 * self.N - 1, generator=g)
        self.rab_time = 0.3 * torch.randn(nb, generator=g)
        self.offs = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int64)
        self.hoffs = np.concatenate([[0], np.cumsum(hist)]).astype(np.int64)
        need = [-(-m // page) for m in hist]
        pool, width = sum(need) + 2, max(need + [0]) + 1
        order = torch.randperm(pool, generator=g).int()
        table = torch.full((B, width), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n

        def poison(*s):  # what lies behind the cached tokens is NaN, or the largest code
            x = torch.full(s, 127 if kind == "int8" else float("nan"))
            return x.to(KINDS[kind]).cuda()
        sc = [None if kind == "bf16" else torch.full((pool, h, page), float("nan")).cuda()
              for _ in range(2)]
        self.cache = hstu.PagedCache(poison(pool, h, page, dqk), poison(pool, h, dv, page),
                                     torch.full((pool, page), -(1 << 60)).cuda(), table.cuda(),
                                     torch.tensor(hist, dtype=torch.int64).cuda(), *sc)
        hstu.hstu_cache_write(self.kc.cuda(), self.vc.cuda(), self.tc.cuda(),
                              torch.from_numpy(self.hoffs).cuda(), self.cache)
        self.parents = torch.tensor([p for x in par for p in x], dtype=torch.int64).cuda()
        self.dev = dict(seq_offsets=torch.from_numpy(self.offs).cuda(), timestamps=self.t.cuda(),
                        rab_pos=self.rab_pos.cuda(), rab_time=self.rab_time.cuda())
        self.max_draft = max(max(nodes), 1)

    def run(self, parents=True, **kw):
        d = self.dev
        a = dict(parents=self.parents if parents else None, max_draft=self.max_draft)
        a.update(kw)
        return hstu.hstu_attn_fwd_tree(self.q, self.k, self.v, d["seq_offsets"], d["timestamps"],
                                       self.cache, d["rab_pos"], d["rab_time"], self.N, **a)

    def want(self, b):
        def f64(x):
            return x.double().cpu().numpy()
        o, e = self.offs[b], self.offs[b + 1]
        s, u = self.hoffs[b], self.hoffs[b + 1]
        return ref.tree(f64(self.q[o:e]), f64(self.k[o:e]), f64(self.v[o:e]),
                        self.t[o:e].numpy(), ref.held(f64(self.kc[s:u]), self.kind),
                        ref.held(f64(self.vc[s:u]), self.kind), self.tc[s:u].numpy(), self.par[b],
                        f64(self.rab_pos), f64(self.rab_time), self.N)

    def check(self, out, users=None):
        for b in range(self.B) if users is None else users:
            want, slack = self.want(b)
            got = out[self.offs[b]:self.offs[b + 1]].double().cpu().numpy()
            err = np.abs(got - want) - (slack + 2.0 ** -8 * np.abs(want))
            assert (err <= 0).all(), f"user {b}: {err.max():.3e} over, row {np.argwhere(err > 0)[0]}"


SHAPES = [
    # hist, nodes, h, d_qk, d_v, page, forest
    ((0,), (1,), 1, 32, 32, 16, "tree"),
    ((1,), (1,), 1, 128, 128, 64, "tree"),
    ((0, 5, 64, 63, 65), (3, 0, 1, 17, 16), 2, 64, 64, 16, "tree"),
    ((300, 0, 127), (33, 64, 5), 4, 64, 64, 32, "tree"),
    ((257, 1000), (65, 130), 3, 128, 128, 64, "comb"),
    ((515, 40), (15, 70), 4, 32, 128, 128, "chain"),
    ((255, 256, 700), (1, 1, 1), 8, 128, 32, 256, "tree"),
    ((100, 3), (200, 31), 5, 64, 32, 64, "flat"),
    ((2100,), (20,), 2, 32, 64, 16, "tree"),
    ((48, 90), (300, 257), 1, 64, 128, 32, "comb"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_against_loops(case, kind):
    hist, nodes, h, dqk, dv, page, shape = SHAPES[case]
    x = Batch(hist, nodes, h, dqk, dv, kind, page, shape, seed=case)
    out = torch.full((x.T, h, dv), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert x.run(out=out) is out
    x.check(out)
    if shape == "flat":  # parents absent: the same bits
        assert torch.equal(out, x.run(parents=False))


@pytest.mark.gpu
def test_many_users():
    """More sequences than a wave has lanes, empty ones among them."""
    r = np.random.default_rng(3)
    hist = tuple(int(v) for v in r.integers(0, 90, 150))
    nodes = tuple(int(v) for v in r.integers(0, 9, 150))
    x = Batch(hist, nodes, 2, 32, 32, "int8", 16, seed=9)
    x.check(x.run())


@pytest.mark.gpu
def test_deep_and_wide():
    """The most drafted tokens a user can have: one chain, and all roots."""
    for shape, seed in (("chain", 1), ("flat", 2)):
        x = Batch((130, 20), (1024, 1023), 1, 32, 32, "e4m3", 64, shape, seed=seed, scale=0.5)
        x.check(x.run())


@pytest.mark.gpu
@pytest.mark.parametrize("nodes", [1, 40])
def test_long_cache(nodes):
    """20001 cached tokens, past the table's N: positions further back take its first entry."""
    x = Batch((20001, 7), (nodes, 1), 2, 64, 64, "e4m3", 256, N=9000, seed=4)
    x.check(x.run())


@pytest.mark.gpu
def test_rows_past_the_end_and_past_max_draft():
    """Rows behind the last sequence, and past max_draft within one, are not
    written; the others are as without them."""
    x = Batch((50, 20), (9, 6), 2, 64, 64, seed=5)
    full = x.run()
    out = torch.full((x.T, 2, 64), 7.0, device="cuda").bfloat16()
    x.run(out=out, max_draft=8)
    rows = torch.tensor([i for i in range(15) if i != 8]).cuda()
    assert (out[8] == 7).all() and torch.equal(out[rows], full[rows])
    x.dev["seq_offsets"] = torch.tensor([0, 9, 12]).cuda()
    out.fill_(7.0)
    x.run(out=out)
    assert (out[12:] == 7).all()
    keep = [i for i in range(9)] + [9, 10, 11]
    assert torch.equal(out[keep], full[keep])


@pytest.mark.gpu
def test_bad_parents_are_roots():
    x = Batch((30, 70), (12, 40), 2, 64, 64, seed=6)
    bad = x.parents.clone()
    for at, value in ((3, 3), (5, 9), (7, -7), (12, 1 << 40), (20, 8)):
        bad[at] = value
    x.par = [bad[:12].tolist(), bad[12:].tolist()]
    x.parents = bad
    x.check(x.run())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_pages_outside_the_pool_are_left_out(kind):
    x = Batch((100, 64), (5, 33), 2, 64, 64, kind, 16, seed=7)
    x.cache.page_table[0, 2] = 1 << 30
    x.cache.page_table[0, 5] = -1
    x.cache.page_table[1, 0] = -5
    for b, gone in ((0, [2, 5]), (1, [0])):
        # left out: the same as values of zero (weights stay finite)
        for pg in gone:
            lo = x.hoffs[b] + 16 * pg
            x.vc[lo:min(lo + 16, int(x.hoffs[b + 1]))] = 0
    x.check(x.run())


@pytest.mark.gpu
@pytest.mark.parametrize("shape", ["tree", "flat"])
def test_what_is_not_seen_changes_no_bit(shape):
    """Infinities and NaN in keys and values of nodes that a row does not see."""
    x = Batch((80, 10), (90, 20), 2, 64, 64, shape=shape, seed=8)
    clean = x.run()
    leaves = [i for i in range(90) if i not in x.par[0]]
    hit = leaves[len(leaves) // 2]
    x.v[hit, :, 3] = float("nan")
    x.v[hit, :, 9] = float("inf")
    x.k[hit, 0, :] = float("inf")
    other = leaves[0]
    x.k[other, :, 1] = float("nan")
    x.v[other] = float("-inf")
    out = x.run()
    rest = torch.tensor([i for i in range(110) if i not in (hit, other)]).cuda()
    assert torch.equal(out[rest], clean[rest])
    assert torch.isnan(out[hit, :, 3]).all() and torch.isnan(out[other].float()).any()
    inner = next(i for i in range(90) if i in x.par[0]) if shape == "tree" else None
    if inner is not None:  # a NaN on the way to the root reaches those below it only
        y = Batch((80, 10), (90, 20), 2, 64, 64, shape=shape, seed=8)
        y.v[inner, 1, 5] = float("nan")
        out = y.run()
        _, ways = ref.depths(y.par[0])
        below = torch.tensor([inner in w for w in ways] + [False] * 20)
        assert torch.equal(torch.isnan(out[:, 1, 5]).cpu(), below)
        mask = torch.ones_like(out, dtype=torch.bool)
        mask[:, 1, 5] = False
        assert torch.equal(out[mask], clean[mask])


@pytest.mark.gpu
def test_infinities_in_the_cache_follow_the_formula():
    """A row held as NaN reaches every drafted token of its user, no other user's."""
    x = Batch((70, 70), (5, 5), 2, 64, 64, "e4m3", seed=10)
    clean = x.run()
    k = torch.randn(1, 2, 64, device="cuda").bfloat16()
    v = k.clone()
    v[0, 1, 4] = float("inf")
    # user 1's token 33
    cache = x.cache
    hstu.hstu_cache_write(k, v, torch.tensor([5]).cuda(), torch.tensor([0, 0, 1]).cuda(), cache,
                          starts=torch.tensor([0, 33]).cuda())
    out = x.run()
    assert torch.equal(out[:5], clean[:5])
    assert torch.isnan(out[5:, 1]).all() and torch.isfinite(out[5:, 0].float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("low", [torch.finfo(torch.float32).min, float("-inf")])
@pytest.mark.parametrize("nodes,hist,N", [((1, 3), (40, 700), None), ((20, 9), (70, 300), None),
                                          ((40, 64), (100, 600), None), ((200, 7), (300, 20), None),
                                          ((300, 1), (260, 5), 2000)])
def test_tables_that_mask(nodes, hist, N, low):
    """Entries of the lowest value, or -inf, in either table or in both: weights of
    0.  The reference takes -200 for them, for which SiLU is below 2^-200."""
    x = Batch(hist, nodes, 2, 32, 32, "int8", 32, "comb", N=N, seed=13, scale=0.5)
    for t in (x.rab_pos, x.rab_time):
        t[torch.rand(t.shape, generator=torch.Generator().manual_seed(14)) < 0.4] = -200.0
    x.rab_pos[x.N - 1] = 0.1  # a token and itself: not masked by the position
    x.rab_time[0] = -200.0    # but by the time
    for name in ("rab_pos", "rab_time"):
        t = getattr(x, name).cuda()
        x.dev[name] = torch.where(t == -200.0, torch.full_like(t, low), t)
    x.check(x.run())
    for name in ("rab_pos", "rab_time"):  # everything masked
        x.dev[name] = torch.full_like(x.dev[name], low)
    assert (x.run() == 0).all() and (x.run(parents=False) == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", list(KINDS))
def test_deterministic_and_independent_of_other_work(kind):
    x = Batch((700, 90, 1500), (20, 1, 64), 4, 64, 64, kind, 64, seed=11)
    a = x.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = x.run()
    c = x.run(ws=torch.full((hstu_ws(x),), 255, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


def hstu_ws(x):
    p = hstu.make_problem(x.B, x.T, x.N, x.h, x.dqk, x.dv, x.rab_time.numel(), hstu.HSTU_BF16)
    return hstu.hstu_attn_fwd_tree_workspace_bytes(p, x.cache, x.max_draft)


@pytest.mark.gpu
def test_two_threads():
    """Calls of two host threads on streams of their own, each with its workspace."""
    xs = [Batch((500, 30), (40, 3), 2, 64, 64, "int8", 32, seed=s) for s in (12, 13)]
    alone = [x.run() for x in xs]
    torch.cuda.synchronize()
    got = [None, None]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(10):
                got[i] = xs[i].run()
            torch.cuda.current_stream().synchronize()
    ts = [threading.Thread(target=work, args=(i,)) for i in (0, 1)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    assert all(torch.equal(a, b) for a, b in zip(alone, got))


@pytest.mark.gpu
def test_captured_and_replayed():
    """One graph over a cache that grows between its replays."""
    x = Batch((600, 130), (16, 9), 4, 64, 64, "e4m3", 64, seed=14)
    out = x.run()
    ws = torch.empty(hstu_ws(x), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.run(out=out, ws=ws)
    for n in (600, 0, 333, 64):
        x.cache.lengths[0] = n
        x.q.mul_(0.9)
        out.fill_(0)
        graph.replay()
        want = x.run()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.gpu
def test_captured_steps():
    """A serving step as one graph: positions, rotary, attention, then all drafted
    tokens (chains) enter the cache; each replay stands behind the one before."""
    lens, drafts, h, d, N = (70, 0, 31), (3, 16, 5), 2, 64, 300
    g = torch.Generator().manual_seed(30)
    T = sum(drafts)
    z = torch.randn(T, 3 * h * d, generator=g).bfloat16().cuda()
    q, k, v = (z[:, i * h * d:(i + 1) * h * d].unflatten(1, (h, d)) for i in range(3))
    ts = torch.randint(0, 1 << 30, (T,), generator=g).cuda()
    rp, rt = (0.1 * torch.randn(n, generator=g).cuda() for n in (2 * N - 1, 32))
    offs = torch.tensor(np.concatenate([[0], np.cumsum(drafts)])).cuda()
    par = torch.tensor([i - 1 for n in drafts for i in range(n)]).cuda()
    freq = torch.from_numpy(hstu.hstu_rotary_frequencies(d)).cuda()
    n_new = torch.tensor(drafts).cuda()

    def fresh():
        cache = hstu.alloc_cache(30, 16, h, d, d, 3, 10, torch.int8)
        cache.page_table.copy_(torch.arange(30).view(3, 10))
        cache.lengths.copy_(torch.tensor(lens))
        ho = torch.tensor(np.concatenate([[0], np.cumsum(lens)])).cuda()
        gen = torch.Generator().manual_seed(31)
        x = torch.randn(sum(lens), h, d, generator=gen).bfloat16().cuda()
        hstu.hstu_cache_write(x, x, torch.arange(sum(lens)).cuda(), ho, cache)
        return cache

    def step(cache):
        pos = hstu.hstu_tree_positions(par, offs, cache.lengths, T, 16)
        qr, kr = hstu.hstu_rotary_fwd(q, k, freq, positions=pos)
        out = hstu.hstu_attn_fwd_tree(qr, kr, v, offs, ts, cache, rp, rt, N, 16, parents=par)
        hstu.hstu_cache_write(kr, v, ts, offs, cache, starts=cache.lengths)
        cache.lengths.add_(n_new)
        return out
    eager, held = fresh(), fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(held)
    for _ in range(4):
        z.mul_(0.9)
        want = step(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(held.lengths, eager.lengths)
    at = torch.tensor(np.concatenate([[0], np.cumsum(eager.lengths.cpu().numpy())])).cuda()
    n = int(at[-1])
    for a, b in zip(hstu.hstu_cache_read(held, at, n), hstu.hstu_cache_read(eager, at, n)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_positions():
    x = Batch((3, 100, 0, 7), (1024, 0, 77, 5), 1, 32, 32, shape="comb", seed=15)
    want = np.concatenate([h + ref.depths(p)[0] for h, p in zip(x.hist, x.par)])
    o, n = x.dev["seq_offsets"], x.cache.lengths
    got = hstu.hstu_tree_positions(x.parents, o, n, x.T, 1024)
    assert np.array_equal(got.cpu().numpy(), want)
    got = hstu.hstu_tree_positions(None, o, n, x.T, 1024)
    assert np.array_equal(got.cpu().numpy(), np.repeat(x.hist, x.nodes))
    got = hstu.hstu_tree_positions(x.parents, o, None, x.T, 1024)
    assert np.array_equal(got.cpu().numpy(), np.concatenate([ref.depths(p)[0] for p in x.par]))
    out = torch.full((x.T,), -9, device="cuda")
    hstu.hstu_tree_positions(x.parents, o, n, x.T, 64, out=out)  # the first 64 of each
    keep = np.concatenate([np.arange(k) < 64 for k in x.nodes])
    assert np.array_equal(out.cpu().numpy(), np.where(keep, want, -9))


@pytest.mark.gpu
def test_served_as_one_sequence():
    """f_1, rotary, cache and tree attention token by token, against one pass of
    the same layer over the whole sequence: chains over a bf16 cache hold the
    same values, so both differ by the rounding of their weights alone."""
    h, d, D, N = 2, 64, 64, 400
    lens, drafts = (301, 64, 20), (7, 64, 1)
    T = sum(lens)
    g = torch.Generator().manual_seed(20)
    x = torch.randn(T, D, generator=g).bfloat16().cuda()
    w1 = (torch.randn(4 * h * d, D, generator=g) / 8).bfloat16().cuda()
    z, _ = hstu.hstu_proj_in_fwd(x, w1, None, h, d, d, want_pre=False)
    u, v, q, k = hstu.split_uvqk(z, h, d, d)
    offs = np.concatenate([[0], np.cumsum(lens)])
    o = torch.tensor(offs).cuda()
    ts = torch.cumsum(torch.randint(0, 5000, (T,), generator=g), 0).cuda()
    rp, rt = (0.1 * torch.randn(n, generator=g).cuda() for n in (2 * N - 1, 64))
    freq = torch.from_numpy(hstu.hstu_rotary_frequencies(48, scaling="linear", factor=2.0)).cuda()
    qr, kr = hstu.hstu_rotary_fwd(q, k, freq, seq_offsets=o)
    whole = hstu.hstu_attn_fwd(qr, kr, v, o, ts, rp, rt, N)

    def rows(take):
        return torch.from_numpy(np.concatenate([np.arange(offs[b], offs[b + 1])[take(b)]
                                                for b in range(3)])).cuda()
    old, new = rows(lambda b: slice(0, lens[b] - drafts[b])), rows(
        lambda b: slice(lens[b] - drafts[b], None))
    hist = [n - m for n, m in zip(lens, drafts)]
    cache = hstu.alloc_cache(24, 32, h, d, d, 3, 10, torch.bfloat16)
    order = torch.randperm(24).int().tolist()
    for b, n in enumerate(lens):
        for i in range(-(-n // 32)):
            cache.page_table[b, i] = order.pop()
    ho = torch.tensor(np.concatenate([[0], np.cumsum(hist)])).cuda()
    hstu.hstu_cache_write(kr[old], v[old], ts[old], ho, cache)
    cache.lengths.copy_(torch.tensor(hist))
    hstu.hstu_cache_validate(cache)
    do = torch.tensor(np.concatenate([[0], np.cumsum(drafts)])).cuda()
    par = torch.tensor([i - 1 for n in drafts for i in range(n)]).cuda()
    n = sum(drafts)
    pos = hstu.hstu_tree_positions(par, do, cache.lengths, n, 64)
    qd, kd = hstu.hstu_rotary_fwd(q[new], k[new], freq, positions=pos)
    assert torch.equal(qd, qr[new]) and torch.equal(kd, kr[new])
    out = hstu.hstu_attn_fwd_tree(qd, kd, v[new], do, ts[new], cache, rp, rt, N, 64, parents=par)
    want = whole[new].float()
    # each side within 2^-8 of sum |weight * value| + 2^-8 |out|: together at
    # most twice that; the sums are bounded with |SiLU(s)| <= |s| + 0.3
    size = torch.zeros_like(want)
    kf, vf, qf = kr.float(), v.float(), qd.float()
    r = 0
    for b in range(3):
        for i in range(drafts[b]):
            upto = offs[b] + hist[b] + i + 1
            s = torch.einsum("hd,khd->hk", qf[r], kf[offs[b]:upto]).abs() + 1.3
            size[r] = torch.einsum("hk,khd->hd", s, vf[offs[b]:upto].abs()) / N
            r += 1
    assert ((out.float() - want).abs() <= 2 * 2.0 ** -8 * (size + want.abs()) * 1.01).all()
    # the accepted tokens enter the cache: one more token over them is a chain's next
    hstu.hstu_cache_write(kd, v[new], ts[new], do, cache, starts=cache.lengths)
    cache.lengths.add_(torch.tensor(drafts).cuda())
    k2, v2, t2 = hstu.hstu_cache_read(cache, o, T)
    assert torch.equal(k2, kr) and torch.equal(v2, v) and torch.equal(t2, ts)
