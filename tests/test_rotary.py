"""Rotary positions: frequencies and refusals (CPU), the turned rows and their
gradients against fp64 loops (GPU).

Tolerance: half a step of the storage type of the result, and for the fp32
arithmetic 2^-21 of |a| + |b| of the pair: sine and cosine are good to two
units of 2^-24, the angle's fp32 fraction of a turn to 2 pi 2^-25, and three
roundings follow."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2402_17152_amd import hstu
from tests import serve_ref as ref

P = ctypes.c_void_p
FAKE = 0x10000  # never read: every call fails before


def test_frequencies():
    f = hstu.hstu_rotary_frequencies(64, 10000.0)
    np.testing.assert_allclose(f, [10000.0 ** (-m / 32) for m in range(32)], rtol=1e-14)
    g = hstu.hstu_rotary_frequencies(64, scaling="linear", factor=4.0)
    np.testing.assert_allclose(g, f / 4, rtol=1e-14)
    g = hstu.hstu_rotary_frequencies(64, scaling="base", factor=4.0)
    assert g[0] == 1.0 and math.isclose(g[-1], f[-1] / 4, rel_tol=1e-12)
    g = hstu.hstu_rotary_frequencies(64, scaling="parts", factor=4.0, original_len=2048)
    turns = 2048 * f / (2 * math.pi)
    assert np.allclose(g[turns >= 32], f[turns >= 32], rtol=1e-14)
    assert np.allclose(g[turns <= 1], f[turns <= 1] / 4, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    keep = (turns[mid] - 1) / 31
    np.testing.assert_allclose(g[mid], f[mid] * (keep + (1 - keep) / 4), rtol=1e-13)
    assert mid.sum() > 3


@pytest.mark.parametrize("kw,needle", [
    (dict(rot_dim=0), "rot_dim"), (dict(rot_dim=7), "rot_dim"), (dict(rot_dim=8, base=0.0), "base"),
    (dict(rot_dim=8, base=math.inf), "base"),
    (dict(rot_dim=8, scaling="linear", factor=0.5), "factor"),
    (dict(rot_dim=8, scaling="linear", factor=math.nan), "factor"),
    (dict(rot_dim=2, scaling="base", factor=2.0), "single pair"),
    (dict(rot_dim=8, scaling="parts", factor=2.0), "original_len"),
    (dict(rot_dim=8, scaling="parts", factor=2.0, original_len=10, low=3, high=3), "low"),
])
def test_frequency_refusals(kw, needle):
    with pytest.raises(hstu.HstuError, match=needle):
        hstu.hstu_rotary_frequencies(**kw)


@pytest.mark.parametrize("kw,status,needle", [
    (dict(rot=3), 1, "rot_dim"), (dict(rot=0), 1, "rot_dim"), (dict(rot=66), 1, "rot_dim"),
    (dict(layout=2), 1, "layout"), (dict(freq=None), 1, "inv_freq"),
    (dict(offs=None, pos=None), 1, "both NULL"), (dict(q=None, k=None), 1, "both NULL"),
    (dict(qo=None), 1, "outputs"), (dict(k=None), 1, "outputs"), (dict(q=FAKE + 8), 1, "aligned"),
    (dict(qs=100), 1, "q_stride"), (dict(ko=FAKE + 4), 1, "aligned"), (dict(ks=132), 1, "multiple"),
    (dict(T=1 << 31), 2, "2\\^31"),
])
@pytest.mark.parametrize("call", ["hstu_rotary_fwd", "hstu_rotary_bwd"])
def test_refusals(call, kw, status, needle):
    a = dict(rot=64, layout=0, freq=FAKE, offs=FAKE, pos=None, q=FAKE, k=FAKE, qo=FAKE, ko=FAKE,
             qs=128, ks=128, T=10)
    a.update(kw)
    p = hstu.make_problem(2, a["T"], 1, 2, 64, 64, 1, hstu.HSTU_BF16)
    st = getattr(hstu.lib, call)(ctypes.byref(p), P(a["offs"]), None, P(a["pos"]), P(a["freq"]),
                                 a["rot"], a["layout"], 1.0, P(a["q"]), a["qs"], P(a["k"]),
                                 a["ks"], P(a["qo"]), P(a["ko"]), None)
    assert st == status
    import re
    assert re.search(needle, hstu.hstu_last_error())


def test_binding_refusals():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    f = torch.ones(32, dtype=torch.float64)
    pos = torch.arange(4)
    for args, kw, err, needle in [
            ((q, q, f.float()), dict(positions=pos), TypeError, "inv_freq"),
            ((q, q[:3], f), dict(positions=pos), ValueError, "k must be"),
            ((q, q.float(), f), dict(positions=pos), TypeError, "k must be"),
            ((q.half(), None, f), dict(positions=pos), TypeError, "unsupported"),
            ((None, None, f), dict(positions=pos), ValueError, "both None"),
            ((q, None, f), dict(positions=pos.int()), TypeError, "positions"),
            ((q, None, f), dict(positions=pos[:2]), ValueError, "positions"),
            ((q.transpose(0, 1).contiguous().transpose(0, 1), None, f), dict(positions=pos),
             ValueError, "contiguous"),
            ((q, None, f), dict(positions=pos, out=(q.float(), None)), ValueError, "q output"),
            ((q, None, f), dict(positions=pos), ValueError, "current device")]:
        with pytest.raises(err, match=needle):
            _with_device(lambda: hstu.hstu_rotary_fwd(*args, **kw))


def _with_device(call):
    """Runs a call that has to be refused before it asks for a stream."""
    saved, hstu._raw_device = hstu._raw_device, lambda: 0
    try:
        return call()
    finally:
        hstu._raw_device = saved


# ------------------------------------------------------------------- GPU

def _half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _check(got, x, pos, freq, interleaved, amplitude=1.0, back=False):
    want, size = ref.rotate(x.double().cpu().numpy(), pos, freq, interleaved, amplitude, back)
    bound = _half_step(got.dtype) * np.abs(want) + 2.0 ** -21 * size
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= bound).all(), f"{(err - bound).max():.3e} over the bound"


def _rows(T, h, d, dtype, seed, strided):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, 2 * h * d + 16, generator=g).to(dtype).cuda()
    if not strided:
        return z[:, :h * d].reshape(T, h, d).contiguous(), z[:, h * d:2 * h * d].reshape(T, h, d)
    return (z[:, 8:8 + h * d].unflatten(1, (h, d)),
            z[:, 8 + h * d:8 + 2 * h * d].unflatten(1, (h, d)))


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,h,d,rot", [(1, 1, 32, 32), (7, 3, 32, 2), (65, 4, 64, 64),
                                       (33, 2, 128, 20), (300, 5, 128, 72), (2, 64, 64, 62),
                                       (4100, 2, 32, 8), (2050, 1, 64, 36)])
def test_positions_given(dtype, interleaved, T, h, d, rot):
    q, k = _rows(T, h, d, dtype, T + rot, strided=rot % 4 == 0)
    g = torch.Generator().manual_seed(T)
    pos = torch.randint(-3, 1 << 20, (T,), generator=g)
    pos[0] = 1 << 24  # far positions keep their angle (to 2^24 * 2^-52 here and there)
    freq = hstu.hstu_rotary_frequencies(rot)
    f = torch.from_numpy(freq).cuda()
    out = [torch.full((T, h, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    got = hstu.hstu_rotary_fwd(q, k, f, positions=pos.cuda(), interleaved=interleaved, out=out)
    assert got[0] is out[0] and got[1] is out[1]
    for y, x in zip(got, (q, k)):
        _check(y, x, pos.numpy(), freq, interleaved)
    back = hstu.hstu_rotary_bwd(q, k, f, positions=pos.cuda(), interleaved=interleaved,
                                amplitude=1.25)
    for y, x in zip(back, (q, k)):
        _check(y, x, pos.numpy(), freq, interleaved, 1.25, True)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [(5,), (0, 1, 0, 40, 3), tuple([1, 2, 0] * 40),
                                     tuple([3] * 4200)])
def test_positions_of_the_batch(lengths):
    """Without positions a token's index counts, candidates sit at the history's
    end, empty sequences and thousands of them included; one of q, k may be absent."""
    g = np.random.default_rng(len(lengths))
    nt = np.array([int(g.integers(0, n + 1)) for n in lengths])
    pos = np.concatenate([np.minimum(np.arange(n), n - c) for n, c in zip(lengths, nt)])
    plain = np.concatenate([np.arange(n) for n in lengths])
    T, h, d = int(sum(lengths)), 2, 32
    q, k = _rows(T, h, d, torch.bfloat16, T, strided=True)
    offs = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int64).cuda()
    freq = hstu.hstu_rotary_frequencies(16)
    f = torch.from_numpy(freq).cuda()
    qo, none = hstu.hstu_rotary_fwd(q, None, f, seq_offsets=offs,
                                    num_targets=torch.tensor(nt).cuda())
    assert none is None
    _check(qo, q, pos, freq, False)
    none, ko = hstu.hstu_rotary_fwd(None, k, f, seq_offsets=offs)
    assert none is None
    _check(ko, k, plain, freq, False)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [70, 5000])
def test_rows_behind_the_last_sequence(T):
    """A batch padded behind its last sequence: the padding is left as it was."""
    q, _ = _rows(T, 2, 32, torch.bfloat16, 8, strided=True)
    f = torch.from_numpy(hstu.hstu_rotary_frequencies(32)).cuda()
    n = T // 2 + 1
    offs = torch.tensor([0, 3, n]).cuda()
    out = torch.full((T, 2, 32), 7.0, device="cuda").bfloat16()
    hstu.hstu_rotary_fwd(q, None, f, seq_offsets=offs, out=(out, None))
    assert (out[n:] == 7).all()
    want, _ = hstu.hstu_rotary_fwd(q[:n], None, f, seq_offsets=offs)
    assert torch.equal(out[:n], want)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place(interleaved):
    q, k = _rows(130, 3, 64, torch.bfloat16, 6, strided=False)
    q, k = q.contiguous(), k.contiguous()
    f = torch.from_numpy(hstu.hstu_rotary_frequencies(40)).cuda()
    pos = torch.arange(130).cuda()
    want = hstu.hstu_rotary_fwd(q, k, f, positions=pos, interleaved=interleaved)
    hstu.hstu_rotary_fwd(q, k, f, positions=pos, interleaved=interleaved, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.gpu
def test_more_workgroups_than_a_row_of_the_grid():
    """2^25 + 33 rows of 32 features (2 GB): the last workgroups lie in a later
    row of the grid."""
    T = (1 << 25) + 33
    x = torch.ones(1, 1, 1, dtype=torch.bfloat16, device="cuda").expand(T, 1, 32).contiguous()
    f = torch.from_numpy(hstu.hstu_rotary_frequencies(32)).cuda()
    pos = torch.arange(T, device="cuda")
    out, _ = hstu.hstu_rotary_fwd(x, None, f, positions=pos)
    for lo in (0, (1 << 25) - 40, T - 70):
        want, _ = hstu.hstu_rotary_fwd(x[lo:lo + 70], None, f, positions=pos[lo:lo + 70])
        assert torch.equal(out[lo:lo + 70], want)


@pytest.mark.gpu
def test_features_behind_the_turned_ones_keep_their_bits():
    x = torch.randn(9, 2, 64, device="cuda").bfloat16()
    x[:, :, 33] = float("nan")
    x[3, 1, 40] = float("inf")
    f = torch.from_numpy(hstu.hstu_rotary_frequencies(32)).cuda()
    y, _ = hstu.hstu_rotary_fwd(x, None, f, positions=torch.arange(9).cuda(), amplitude=3.0)
    assert torch.equal(y[..., 32:].view(torch.int16), x[..., 32:].view(torch.int16))
    assert torch.isfinite(y[..., :32].float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(interleaved):
    """<y, w> changes by <dx, e> for small steps e: the map is linear, so the
    difference of two fp32 passes is exact up to their rounding."""
    T, h, d = 17, 2, 64
    g = torch.Generator().manual_seed(3)
    x, w, e = (torch.randn(T, h, d, generator=g).cuda() for _ in range(3))
    offs = torch.tensor([0, 4, 17]).cuda()
    f = torch.from_numpy(hstu.hstu_rotary_frequencies(40)).cuda()
    kw = dict(seq_offsets=offs, interleaved=interleaved, amplitude=0.7)
    dx, _ = hstu.hstu_rotary_bwd(w, None, f, **kw)
    y0, _ = hstu.hstu_rotary_fwd(x - e, None, f, **kw)
    y1, _ = hstu.hstu_rotary_fwd(x + e, None, f, **kw)
    lhs = ((y1.double() - y0.double()) / 2 * w.double()).sum().item()
    rhs = (dx.double() * e.double()).sum().item()
    size = (w.abs().double() * (x.abs() + e.abs()).double()).sum().item()
    assert abs(lhs - rhs) <= size * 8 * 2.0 ** -24 * 4


@pytest.mark.gpu
def test_captured_and_replayed():
    T, h, d = 300, 2, 64
    q, k = _rows(T, h, d, torch.bfloat16, 1, strided=True)
    pos = torch.arange(T).cuda()
    f = torch.from_numpy(hstu.hstu_rotary_frequencies(64)).cuda()
    out = hstu.hstu_rotary_fwd(q, k, f, positions=pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hstu.hstu_rotary_fwd(q, k, f, positions=pos, out=out)
    for step in range(3):
        pos += 100 * step
        q.mul_(0.5)
        graph.replay()
        want = hstu.hstu_rotary_fwd(q, k, f, positions=pos)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
