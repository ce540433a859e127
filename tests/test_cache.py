"""The paged cache: refusals (CPU), codes, scales and rows read back against the
fp64 definition, and what a write must leave alone (GPU).  Codes and scales are
exact by definition, so is what is read back: code * scale in fp32, rounded once."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2402_17152_amd import hstu
from tests import serve_ref as ref

P = ctypes.c_void_p
FAKE = 0x10000  # never read: every call fails before
KINDS = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def _desc(**kw):
    a = dict(num_pages=8, page_size=64, max_pages=4, dtype=hstu.HSTU_CACHE_E4M3, k=FAKE, v=FAKE,
             k_scale=FAKE, v_scale=FAKE, timestamps=FAKE, page_table=FAKE, lengths=FAKE)
    a.update(kw)
    return hstu.CacheDesc(**a)


def _problem(**kw):
    a = dict(num_seqs=2, total_tokens=10, max_seq_len=1, num_heads=2, d_qk=64, d_v=32,
             num_time_buckets=1, dtype=hstu.HSTU_BF16)
    a.update(kw)
    return hstu.make_problem(**a)


def _write(p, c, offs=FAKE, ts=FAKE, k=FAKE, ks=128, v=FAKE, vs=64):
    return hstu.lib.hstu_cache_write(ctypes.byref(p), None if c is None else ctypes.byref(c),
                                     P(offs), None, P(ts), P(k), ks, P(v), vs, None)


def _read(p, c, offs=FAKE, k=FAKE, v=FAKE):
    return hstu.lib.hstu_cache_read(ctypes.byref(p), None if c is None else ctypes.byref(c),
                                    P(offs), None, P(k), P(v), None, None)


BAD_CACHES = [
    (dict(num_pages=0), 1, "num_pages"), (dict(num_pages=1 << 31), 1, "num_pages"),
    (dict(max_pages=0), 1, "max_pages"), (dict(page_size=8), 2, "page_size"),
    (dict(page_size=48), 2, "page_size"), (dict(page_size=512), 2, "page_size"),
    (dict(page_size=0), 2, "page_size"), (dict(dtype=3), 1, "dtype"), (dict(k=None), 1, "cache k"),
    (dict(v=FAKE + 8), 1, "cache v"), (dict(k_scale=None), 1, "k_scale"),
    (dict(v_scale=FAKE + 4), 1, "v_scale"), (dict(timestamps=None), 1, "timestamps"),
    (dict(page_table=None), 1, "page_table"),
]


@pytest.mark.parametrize("kw,status,needle", BAD_CACHES)
def test_cache_refusals(kw, status, needle):
    for call in (_write, _read):
        assert call(_problem(), _desc(**kw)) == status
        assert needle in hstu.hstu_last_error()
    assert hstu.lib.hstu_cache_validate(ctypes.byref(_problem()), ctypes.byref(_desc(**kw)),
                                        None) == status


def test_call_refusals():
    p, c = _problem(), _desc()
    for call, status, needle in [
            (lambda: _write(p, None), 1, "cache is NULL"),
            (lambda: _write(_problem(d_qk=48), c), 2, "d_qk"),
            (lambda: _write(p, c, offs=None), 1, "seq_offsets"),
            (lambda: _write(p, c, ts=None), 1, "timestamps"),
            (lambda: _write(p, c, k=None), 1, "k is NULL"),
            (lambda: _write(p, c, ks=64), 1, "k_stride"),
            (lambda: _write(p, c, v=FAKE + 2), 1, "aligned"),
            (lambda: _write(p, c, vs=68), 1, "multiple of 16"),
            (lambda: _read(p, c, offs=None), 1, "seq_offsets"),
            (lambda: _read(p, c, k=None), 1, "k is NULL"),
            (lambda: _read(p, c, v=FAKE + 8), 1, "aligned"),
            (lambda: _read(p, _desc(lengths=None)), 1, "lengths")]:
        assert call() == status
        assert needle in hstu.hstu_last_error()
    # nothing to do: no pointer is looked at
    assert _write(_problem(total_tokens=0), c, ts=None, k=None, v=None) == 0
    assert _read(_problem(total_tokens=0), c, k=None, v=None) == 0


def _arrays(kind, pages=5, h=2, page=16, dqk=32, dv=64, B=3, width=4, device="cpu"):
    t = KINDS[kind]
    sc = [None if kind == "bf16" else torch.ones(pages, h, page, device=device) for _ in range(2)]
    return dict(k=torch.zeros(pages, h, page, dqk, device=device).to(t),
                v=torch.zeros(pages, h, dv, page, device=device).to(t),
                timestamps=torch.zeros(pages, page, dtype=torch.int64, device=device),
                page_table=torch.zeros(B, width, dtype=torch.int32, device=device),
                lengths=torch.zeros(B, dtype=torch.int64, device=device), k_scale=sc[0],
                v_scale=sc[1])


@pytest.mark.parametrize("kw,err,needle", [
    (dict(k=torch.zeros(5, 2, 16, 32)), TypeError, "not supported"),
    (dict(v=torch.zeros(5, 2, 64, 16, dtype=torch.bfloat16)), TypeError, "not supported"),
    (dict(v=torch.zeros(5, 2, 16, 64, dtype=torch.int8)), ValueError, "v must be"),
    (dict(timestamps=torch.zeros(5, 8, dtype=torch.int64)), ValueError, "timestamps"),
    (dict(timestamps=torch.zeros(5, 16)), TypeError, "timestamps"),
    (dict(page_table=torch.zeros(3, 4, dtype=torch.int64)), TypeError, "page_table"),
    (dict(page_table=torch.zeros(4, 3, dtype=torch.int32).t()), ValueError, "contiguous"),
    (dict(lengths=torch.zeros(2, dtype=torch.int64)), ValueError, "lengths"),
    (dict(k_scale=None), ValueError, "scales"), (dict(v_scale=None), ValueError, "scales"),
    (dict(k_scale=torch.ones(5, 16, 2)), ValueError, "scales"),
    (dict(k_scale=torch.ones(5, 2, 16).double()), TypeError, "k_scale"),
])
def test_paged_cache_refusals(kw, err, needle):
    a = _arrays("int8")
    hstu.PagedCache(**a)
    a.update(kw)
    with pytest.raises(err, match=needle):
        hstu.PagedCache(**a)
    b = _arrays("bf16")
    hstu.PagedCache(**b)
    with pytest.raises(ValueError, match="scales"):
        hstu.PagedCache(**{**b, "k_scale": torch.ones(5, 2, 16)})


def test_reference_quantiser():
    """The oracle's codes on values worked out by hand."""
    c, s = ref.quantise([[448.0, -1.0, 17.0, 0.0], [2.0, 0.0, 0.0, -2.0]], "e4m3")
    assert s.tolist() == [1.0, 2.0 ** -7] and c[0].tolist() == [448.0, -1.0, 16.0, 0.0]
    assert c[1].tolist() == [256.0, 0.0, 0.0, -256.0]
    c, s = ref.quantise([[449.0, 1.0, 0.0], [127.0, 63.5, -62.5]], "e4m3")
    assert s[0] == 2.0 and c[0].tolist() == [224.0, 0.5, 0.0]
    c, s = ref.quantise([[127.0, 63.5, -62.5], [0.0, 0.0, 0.0], [1.0, np.inf, 2.0]], "int8")
    # 127 times the fp32 number nearest to 1/127, which is below it, rounds to 1
    assert c[0].tolist() == [127.0, 64.0, -62.0] and s[0] == 1.0
    assert s[1] == 1.0 and np.isnan(s[2]) and not c[2].any()
    assert len(ref.e4m3_values()) == 127 and ref.e4m3_values()[-1] == 448.0


# ------------------------------------------------------------------- GPU

class Fill:
    """A cache with known content everywhere, and its state before a call."""

    def __init__(self, kind, page, h, dqk, dv, caps, seed=0):
        g = torch.Generator().manual_seed(seed)
        need = [-(-c // page) for c in caps]
        pool, width = sum(need) + 3, max(need + [1]) + 1
        order = torch.randperm(pool, generator=g).int()
        table = torch.full((len(caps), width), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        t = KINDS[kind]

        def fill(*shape):
            x = torch.randn(shape, generator=g) * 20
            return (x.round().clamp(-127, 127) if kind == "int8" else x).to(t).cuda()
        self.kind, self.page, self.h = kind, page, h
        sc = [None if kind == "bf16" else torch.rand(pool, h, page, generator=g).cuda()
              for _ in range(2)]
        self.cache = hstu.PagedCache(
            fill(pool, h, page, dqk), fill(pool, h, dv, page),
            torch.randint(0, 1 << 40, (pool, page), generator=g).cuda(), table.cuda(),
            torch.tensor(caps, dtype=torch.int64).cuda(), *sc)
        self.table = table.numpy()
        self.before = self.state()

    def state(self):
        """k, v codes as numbers [pool, h, page, d], scales, timestamps."""
        c = self.cache
        k, v = (x.float().cpu().numpy().astype(np.float64) for x in (c.k, c.v))
        sc = [None if s is None else s.cpu().numpy().astype(np.float64)
              for s in (c.k_scale, c.v_scale)]
        return [k, v.swapaxes(2, 3).copy(), sc[0], sc[1], c.timestamps.cpu().numpy().copy()]

    def place(self, b, t):
        return int(self.table[b, t // self.page]), t % self.page


def _rows(T, h, dqk, dv, dtype, seed):
    """Rows as views of one projection output, with the values where a code
    can go wrong: ties, zeros, tiny, huge, one infinity, one NaN."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, h * (dqk + dv) + 8, generator=g)
    z *= torch.exp2(torch.randint(-30, 30, (T, 1), generator=g).float())
    k, v = z[:, 8:8 + h * dqk].unflatten(1, (h, dqk)), z[:, 8 + h * dqk:].unflatten(1, (h, dv))
    k[0] = torch.arange(dqk) - 0.5               # int8 ties where the scale is 1
    k[0, :, -1] = 127.0
    v[0] = torch.linspace(-448, 448, dv)
    if T > 6:
        k[1] = 0.0
        k[2] *= 1e-36 / k[2].abs().max()         # below 2^-100
        v[2, :, 0] = 3.0e38
        k[3, 0, 5] = float("inf")
        v[4, -1, 1] = float("nan")
        v[5] = 2.0 ** torch.arange(dv)[None].clamp(max=60).float() * 2.0 ** -40
        k[6, :, 1:] = 0.0
    z = z.to(dtype).cuda()
    return (z[:, 8:8 + h * dqk].unflatten(1, (h, dqk)),
            z[:, 8 + h * dqk:].unflatten(1, (h, dv)))


def _expect_write(f, k, v, ts, offs, starts):
    """The state after a write, by the definition."""
    st = f.state()
    k, v = k.double().cpu().numpy(), v.double().cpu().numpy()
    if f.kind == "bf16":
        rows = [(ref.held(k, "bf16"), None), (ref.held(v, "bf16"), None)]
    else:
        rows = [ref.quantise(k, f.kind), ref.quantise(v, f.kind)]
    for b in range(len(offs) - 1):
        for i in range(offs[b + 1] - offs[b]):
            t, r = starts[b] + i, offs[b] + i
            if t < 0 or t >= f.table.shape[1] * f.page or f.table[b, t // f.page] < 0:
                continue
            page, at = f.place(b, t)
            for side in (0, 1):
                st[side][page, :, at] = rows[side][0][r]
                if rows[side][1] is not None:
                    st[2 + side][page, :, at] = rows[side][1][r]
            st[4][page, at] = ts[r]
    return st


CASES = [
    # (page, h, d_qk, d_v, rows per user, first position per user)
    (16, 1, 32, 32, (1,), (0,)),
    (16, 3, 32, 64, (5, 0, 40, 1), (3, 0, 15, 63)),
    (32, 2, 64, 32, (33, 64, 7), (31, 0, 100)),
    (64, 4, 128, 128, (130, 1), (1, 127)),
    (128, 2, 128, 32, (300, 65, 0, 2), (0, 63, 5, 126)),
    (256, 1, 64, 128, (257, 70), (200, 250)),
    (32, 2, 32, 128, tuple([2, 0, 3] * 30), tuple(range(90))),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("case", range(len(CASES)))
def test_write_and_read(case, kind, dtype):
    page, h, dqk, dv, lens, starts = CASES[case]
    f = Fill(kind, page, h, dqk, dv, [s + n for s, n in zip(starts, lens)], seed=case)
    T = sum(lens)
    offs = np.concatenate([[0], np.cumsum(lens)])
    k, v = _rows(T, h, dqk, dv, dtype, 10 + case)
    ts = torch.randint(0, 1 << 61, (T,)).cuda()
    o, s = torch.tensor(offs).cuda(), torch.tensor(starts).cuda()
    want = _expect_write(f, k, v, ts.cpu().numpy(), offs, starts)
    hstu.hstu_cache_write(k, v, ts, o, f.cache, starts=s)
    for name, a, b in zip(("k", "v", "k_scale", "v_scale", "timestamps"), f.state(), want):
        if a is not None:
            assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f"), name
    for out_type in (torch.bfloat16, torch.float32):
        rk, rv, rt = hstu.hstu_cache_read(f.cache, o, T, starts=s, dtype=out_type)
        assert torch.equal(rt, ts)
        for got, x in ((rk, k), (rv, v)):
            x = x.double().cpu().numpy()
            if kind == "bf16":
                y = torch.from_numpy(ref.held(x, "bf16"))
            else:
                c, sc = ref.quantise(x, kind)
                y = torch.from_numpy(c.astype(np.float32) * sc.astype(np.float32)[..., None])
            y = y.float().to(out_type)
            assert torch.equal(torch.nan_to_num(got.cpu().float(), nan=-12345.0),
                               torch.nan_to_num(y.float(), nan=-12345.0))


@pytest.mark.gpu
def test_every_code_of_a_row():
    """All ties and neighbours of ties of both 8-bit types, at scales that are
    not powers of two, from fp32 rows."""
    g = torch.Generator().manual_seed(0)
    for kind in ("int8", "e4m3"):
        tops = torch.rand(64, generator=g) * 4 + 0.1
        rows = torch.zeros(64, 1, 128)
        for r, top in enumerate(tops.tolist()):
            top = float(np.float32(top))
            s = ref.quantise([[top]], kind)[1][0]
            if kind == "int8":
                mid = (np.arange(1, 127) - 0.5) * s
            else:
                t = ref.e4m3_values()
                mid = (t[:-1] + t[1:]) / 2 * s
                mid = mid[mid <= top][-126:]
            mid = np.resize(mid, 126).astype(np.float32)
            if r % 3:  # the fp32 neighbours of the ties
                mid = np.nextafter(mid, np.float32(0 if r % 3 == 1 else 1e9))
            rows[r, 0, 0] = top
            rows[r, 0, 1:127] = torch.from_numpy(mid) * (1 if r % 2 else -1)
        rows = rows.clamp(-tops[:, None, None].float(), tops[:, None, None].float())
        f = Fill(kind, 64, 1, 128, 128, [64])
        offs = torch.tensor([0, 64]).cuda()
        ts = torch.arange(64).cuda()
        want = _expect_write(f, rows, rows, ts.cpu().numpy(), [0, 64], [0])
        hstu.hstu_cache_write(rows.cuda(), rows.cuda(), ts, offs, f.cache)
        for a, b in zip(f.state(), want):
            assert np.array_equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["e4m3", "bf16"])
def test_positions_and_pages_out_of_range(kind):
    """Writes there are dropped, reads give zeros, neighbours keep their bits;
    rows behind the last sequence stay as they were."""
    f = Fill(kind, 16, 2, 32, 32, [40, 40, 40, 40], seed=5)
    f.cache.page_table[1, 0] = 1 << 30           # outside the pool
    f.table[1, 0] = -1
    lens, starts = (20, 20, 20, 20), (-5, 0, 40, 1 << 62)
    T = 80
    offs = np.concatenate([[0], np.cumsum(lens)])
    k, v = _rows(T + 4, 2, 32, 32, torch.bfloat16, 3)
    ts = torch.arange(T + 4).cuda()
    o, s = torch.tensor(offs).cuda(), torch.tensor(starts).cuda()
    want = _expect_write(f, k, v, ts.cpu().numpy(), offs, starts)
    hstu.hstu_cache_write(k, v, ts, o, f.cache, starts=s)
    for a, b in zip(f.state(), want):
        if a is not None:
            assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f")
    with pytest.raises(hstu.HstuError, match="page_table\\[1\\]\\[0\\]"):
        hstu.hstu_cache_validate(f.cache)
    out = (torch.full((T + 4, 2, 32), 9.0, device="cuda").bfloat16(),
           torch.full((T + 4, 2, 32), 9.0, device="cuda").bfloat16(),
           torch.full((T + 4,), 9, device="cuda"))
    hstu.hstu_cache_read(f.cache, o, T + 4, starts=s, out=out)
    rk, rv, rt = (x.cpu() for x in out)
    assert (rk[T:] == 9).all() and (rv[T:] == 9).all() and (rt[T:] == 9).all()
    assert not rk[:5].any() and not rt[:5].any()          # positions -5 .. -1
    assert rt[5:20].tolist() == ts[5:20].tolist()
    assert not rk[20:36].any() and not rv[20:36].any()    # the page outside
    assert rt[36:40].tolist() == ts[36:40].tolist()
    assert not rk[40:80].any() and not rv[40:80].any() and not rt[40:80].any()


@pytest.mark.gpu
def test_validate():
    f = Fill("int8", 16, 1, 32, 32, [17, 0, 5])
    hstu.hstu_cache_validate(f.cache)
    f.cache.lengths[1] = f.cache.page_table.shape[1] * 16 + 1
    with pytest.raises(hstu.HstuError, match="lengths\\[1\\]"):
        hstu.hstu_cache_validate(f.cache)
    f.cache.lengths[1] = -1
    with pytest.raises(hstu.HstuError, match="lengths\\[1\\]"):
        hstu.hstu_cache_validate(f.cache)


@pytest.mark.gpu
def test_pool_past_32_bits():
    """A pool of 4.5 GB of values: offsets of its last pages pass 2^32 bytes, and
    2^31 elements."""
    pages, h, page, d = 70000, 4, 128, 128
    k = torch.empty(pages, h, page, d, dtype=torch.int8, device="cuda")
    v = torch.empty(pages, h, d, page, dtype=torch.int8, device="cuda")
    sc = [torch.empty(pages, h, page, device="cuda") for _ in range(2)]
    table = torch.tensor([[pages - 1, 0, pages // 2]], dtype=torch.int32, device="cuda")
    cache = hstu.PagedCache(k, v, torch.empty(pages, page, dtype=torch.int64, device="cuda"),
                            table, torch.tensor([300]).cuda(), *sc)
    x = torch.randn(300, h, d, device="cuda").bfloat16()
    y = torch.randn(300, h, d, device="cuda").bfloat16()
    ts = torch.arange(300).cuda()
    offs = torch.tensor([0, 300]).cuda()
    hstu.hstu_cache_write(x, y, ts, offs, cache)
    rk, rv, rt = hstu.hstu_cache_read(cache, offs, 300, dtype=torch.float32)
    for got, src in ((rk, x), (rv, y)):
        c, s = ref.quantise(src.double().cpu().numpy(), "int8")
        want = c.astype(np.float32) * s.astype(np.float32)[..., None]
        assert np.array_equal(got.cpu().numpy(), want)
    assert torch.equal(rt, ts)


@pytest.mark.gpu
def test_captured_and_replayed():
    f = Fill("e4m3", 32, 2, 64, 64, [64, 64])
    offs = torch.tensor([0, 1, 2]).cuda()
    starts = torch.zeros(2, dtype=torch.int64, device="cuda")
    k = torch.randn(2, 2, 64, device="cuda").bfloat16()
    ts = torch.zeros(2, dtype=torch.int64, device="cuda")
    out = hstu.hstu_cache_read(f.cache, offs, 2, starts=starts)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hstu.hstu_cache_write(k, k, ts, offs, f.cache, starts=starts)
        hstu.hstu_cache_read(f.cache, offs, 2, starts=starts, out=out)
    for step in range(4):
        starts.fill_(17 * step)
        ts.fill_(step)
        k.normal_()
        graph.replay()
        torch.cuda.synchronize()
        want = torch.from_numpy(ref.held(k.double().cpu().numpy(), "e4m3")).bfloat16()
        assert torch.equal(out[0].cpu(), want) and torch.equal(out[1].cpu(), want)
        assert out[2].tolist() == [step, step]
