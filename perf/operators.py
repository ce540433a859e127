"""The operators of token-by-token serving and of rotary positions, for timing
and for comparing outputs.

Three groups, which a program uses one after another: rotary positions of Q
and K with their gradient (`rotary`), the paged cache of a user's keys and
values, quantised as it is written, and its reading back (`cache`), and the
attention of a tree of drafted tokens over such a cache (`tree`); `step` is a
serving step that chains them.  With `own` false a case is computed in plain
torch operations, with `own` true by the library's calls, from the same inputs.

Layout of the paged cache: keys [pages][h][page][d_qk], values transposed,
[pages][h][d_v][page], fp32 scales [pages][h][page] of quantised rows (a row
is one token of one head), int64 timestamps [pages][page].  Token t of user b
lies in page page_table[b][t // page] at place t % page.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TIME_ORIGIN = 1_700_000_000
GAP_MEAN_S = 600.0
RAB_STD = 0.02
TIME_BUCKETS = 128
ROTARY_BASE = 10000.0
MAX_BYTES = 2.4e8      # cost bounds of a drawn case, below the largest listed one
MAX_FLOPS = 5.0e10
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn,
         "int8": torch.int8}


def listed():
    """The calls in use, smallest to largest of each kind."""
    return [
        # Rotary positions of one decoding step: a token for each of 64 users.
        {"name": "rotary_token", "op": "rotary", "way": "fwd", "dtype": "bf16", "batch": 64,
         "lo": 1, "hi": 1, "heads": 4, "d_qk": 128, "d_v": 128, "rot": 128,
         "interleaved": False, "scaling": 1.0, "far": 8192},
        # The training batch (skewed lengths up to 4096, eight heads of 64),
        # Q and K as views of the fused projection output.
        {"name": "rotary_train", "op": "rotary", "way": "fwd", "dtype": "bf16", "batch": 64,
         "lo": 64, "hi": 4096, "heads": 8, "d_qk": 64, "d_v": 64, "rot": 64,
         "interleaved": False, "scaling": 1.0, "far": 0},
        # Gradients on long histories: interleaved pairs, half of each head,
        # frequencies stretched four times for longer contexts.
        {"name": "rotary_bwd_long", "op": "rotary", "way": "bwd", "dtype": "bf16", "batch": 8,
         "lo": 4096, "hi": 8192, "heads": 4, "d_qk": 128, "d_v": 128, "rot": 64,
         "interleaved": True, "scaling": 4.0, "far": 0},
        # The smallest training batch, fp32.
        {"name": "rotary_bwd_fp32", "op": "rotary", "way": "bwd", "dtype": "f32", "batch": 4,
         "lo": 16, "hi": 128, "heads": 2, "d_qk": 32, "d_v": 32, "rot": 32,
         "interleaved": False, "scaling": 1.0, "far": 0},
        # Histories enter the cache and are read back (hand-over to another
        # worker): 16 users of up to 2048 tokens, 8-bit floating point.
        {"name": "cache_prompt_e4m3", "op": "cache", "write": True, "dtype": "bf16",
         "cache": "e4m3", "page": 64, "batch": 16, "lo": 1024, "hi": 2048, "start": 0,
         "heads": 4, "d_qk": 128, "d_v": 128},
        # One new token for each of 64 users, behind what they have, and read back.
        {"name": "cache_append_int8", "op": "cache", "write": True, "dtype": "bf16",
         "cache": "int8", "page": 16, "batch": 64, "lo": 1, "hi": 1, "start": 2000,
         "heads": 8, "d_qk": 64, "d_v": 64},
        # Long cached histories read back whole.
        {"name": "cache_read_int8", "op": "cache", "write": False, "dtype": "bf16",
         "cache": "int8", "page": 128, "batch": 8, "lo": 4096, "hi": 8192, "start": 0,
         "heads": 4, "d_qk": 128, "d_v": 128},
        # One token for each of 16 users over short histories: latency.
        {"name": "tree_token_bf16", "op": "tree", "cache": "bf16", "page": 32, "batch": 16,
         "lo": 20, "hi": 1024, "nodes_lo": 1, "nodes_hi": 1, "shape": "chain", "heads": 4,
         "d_qk": 64, "d_v": 64, "max_len": 1100},
        # Trees of up to 64 drafted tokens over the encoder's long histories.
        {"name": "tree_draft_e4m3", "op": "tree", "cache": "e4m3", "page": 64, "batch": 16,
         "lo": 4096, "hi": 8000, "nodes_lo": 40, "nodes_hi": 64, "shape": "tree", "heads": 4,
         "d_qk": 128, "d_v": 128, "max_len": 8192},
        # One user with a lifetime of actions, seven drafted tokens.
        {"name": "tree_long_int8", "op": "tree", "cache": "int8", "page": 256, "batch": 1,
         "lo": 60001, "hi": 60001, "nodes_lo": 7, "nodes_hi": 7, "shape": "tree", "heads": 2,
         "d_qk": 128, "d_v": 128, "max_len": 65536},
        # Ranking: a thousand candidates for each user, no drafted history.
        {"name": "tree_rank_bf16", "op": "tree", "cache": "bf16", "page": 64, "batch": 16,
         "lo": 1024, "hi": 2048, "nodes_lo": 1000, "nodes_hi": 1024, "shape": "flat", "heads": 4,
         "d_qk": 128, "d_v": 128, "max_len": 4096},
        # A serving step: the accepted tokens of the last step enter the
        # cache, then trees of 16 drafted tokens are rotated and attend.
        {"name": "step_e4m3", "op": "step", "cache": "e4m3", "page": 64, "batch": 32,
         "lo": 1000, "hi": 4000, "nodes_lo": 8, "nodes_hi": 16, "shape": "tree", "heads": 8,
         "d_qk": 64, "d_v": 64, "max_len": 4096, "accepted": 4, "rot": 64,
         "interleaved": False, "scaling": 1.0},
    ]


# ------------------------------------------------------------------ shapes

def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _rng(case):
    return random.Random("/".join(str(case.get(k)) for k in ("op", "batch", "lo", "hi", "nodes_lo",
                                                             "nodes_hi", "shape", "start")))


def _lengths(case):
    """Tokens per user (rotary, cache: the rows; tree, step: the history)."""
    rng = _rng(case)
    if case["op"] == "rotary" and case["hi"] >= 16 * case["lo"]:
        return [_log_int(rng, case["lo"], case["hi"]) for _ in range(case["batch"])]
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]


def _starts(case):
    rng = random.Random("starts/%d/%d" % (case["batch"], case["start"]))
    return [rng.randint(case["start"] // 2, case["start"]) for _ in range(case["batch"])]


def _trees(case):
    """(nodes, parents) of each user: parents as a list, -1 at a root."""
    rng = random.Random("nodes/" + str(_rng(case).random()))
    out = []
    for _ in range(case["batch"]):
        n = rng.randint(case["nodes_lo"], case["nodes_hi"])
        if case["shape"] == "flat":
            par = [-1] * n
        elif case["shape"] == "chain":
            par = list(range(-1, n - 1))
        else:  # a node follows one of the eight before it, or starts a branch of its own
            par = [max(-1, rng.randint(i - 8, i - 1)) for i in range(n)]
        out.append((n, par))
    return out


def _depths(par):
    d = []
    for p in par:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _accepted(case):
    rng = random.Random("accepted/%d" % case["batch"])
    return [rng.randint(1, case["accepted"]) for _ in range(case["batch"])]


def work(case):
    """What a pass cannot do without."""
    h, dqk, dv = case["heads"], case["d_qk"], case["d_v"]
    if case["op"] == "rotary":
        T, e = sum(_lengths(case)), 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 4.0 * T * h * dqk * e + 8.0 * T, "flops": 6.0 * T * h * case["rot"]}
    ce = 2 if case["cache"] == "bf16" else 1
    row = h * (dqk + dv) * ce + (0 if ce == 2 else 8 * h) + 8  # of the cache, scales and time
    if case["op"] == "cache":
        T, e = sum(_lengths(case)), 2 if case["dtype"] == "bf16" else 4
        full = h * (dqk + dv) * e + 8
        n = 2 * (row + full) if case["write"] else row + full
        return {"bytes": float(T * n), "flops": 4.0 * T * h * (dqk + dv)}
    hist, trees = _lengths(case), _trees(case)
    T = sum(n for n, _ in trees)
    pairs = sum(n * m for (n, _), m in zip(trees, hist)) + sum(
        sum(d + 1 for d in _depths(par)) for _, par in trees)
    b = sum(hist) * row + T * h * (2 * dqk + 2 * dv) * 2 + 16 * T
    if case["op"] == "step":
        acc = sum(_accepted(case))
        b += acc * (row + h * (dqk + dv) * 2)
        pairs += sum(n * a for (n, _), a in zip(trees, _accepted(case)))
    return {"bytes": float(b), "flops": 2.0 * (dqk + dv) * h * pairs}


def _shrink(case):
    while case["batch"] > 1:
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS:
            return case
        case["batch"] //= 2
    w = work(case)
    if "nodes_hi" in case and w["flops"] > MAX_FLOPS:
        case["nodes_hi"] = 256
        case["nodes_lo"] = min(case["nodes_lo"], 256)
    return case


def draw(rng):
    """One more case of the ranges that the listed ones stand for."""
    op = rng.choice(["rotary", "rotary", "cache", "cache", "tree", "tree", "tree", "step"])
    d = rng.choice([32, 64, 128])
    case = {"op": op, "heads": rng.choice([1, 2, 3, 4, 5, 8]), "d_qk": d,
            "d_v": d if rng.random() < 0.7 else rng.choice([32, 64, 128])}
    if op in ("rotary", "step"):
        case |= {"rot": d if rng.random() < 0.5 else 2 * rng.randint(1, d // 2),
                 "interleaved": rng.random() < 0.5, "scaling": rng.choice([1.0, 1.0, 2.0, 8.0])}
    if op in ("rotary", "cache"):
        hi = _log_int(rng, 1, 8192)
        case |= {"dtype": rng.choice(["bf16", "bf16", "f32"]), "batch": _log_int(rng, 1, 64),
                 "lo": rng.randint(1, hi), "hi": hi}
    if op == "rotary":
        case |= {"way": rng.choice(["fwd", "bwd"]), "far": rng.choice([0, _log_int(rng, 64, 65536)])}
        return _shrink(case)
    case |= {"cache": rng.choice(["bf16", "e4m3", "e4m3", "int8"]),
             "page": rng.choice([16, 32, 64, 128, 256])}
    if op == "cache":
        case |= {"write": rng.random() < 0.6, "start": rng.choice([0, _log_int(rng, 1, 4096)])}
        return _shrink(case)
    hi, nodes = _log_int(rng, 1, 32768), _log_int(rng, 1, 300)
    case |= {"batch": _log_int(rng, 1, 64), "lo": rng.randint(0, hi), "hi": hi,
             "nodes_lo": rng.randint(1, nodes), "nodes_hi": nodes,
             "shape": rng.choice(["tree", "tree", "chain", "flat"]),
             "max_len": hi + nodes + rng.randint(4, 64)}
    if op == "step":
        case["accepted"] = rng.randint(1, 8)
        case["max_len"] += 8
    return _shrink(case)


# ------------------------------------------------------------------ inputs

def _offsets(lengths, device="cuda"):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int64, device=device)


def _frequencies(case):
    """Inverse frequencies in fp64; the base grows with the stretch, so that
    the slowest pair turns `scaling` times slower and the fastest as before."""
    rot = case["rot"]
    base = ROTARY_BASE
    if case["scaling"] != 1.0 and rot > 2:
        base *= case["scaling"] ** (rot / (rot - 2))
    m = torch.arange(rot // 2, dtype=torch.float64)
    return torch.pow(torch.tensor(base, dtype=torch.float64), -2.0 * m / rot).cuda()


def _silu_rows(gen, *shape, dtype=torch.float32):
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x * torch.sigmoid(x)).to(dtype)


def _fused(gen, T, h, dqk, dv, dtype):
    """U, V, Q, K as views of one projection output [T][U|V|Q|K]."""
    z = _silu_rows(gen, T, 2 * h * (dqk + dv), dtype=dtype)
    cut = [h * dv, 2 * h * dv, 2 * h * dv + h * dqk]
    return (z[:, cut[0]:cut[1]].unflatten(1, (h, dv)), z[:, cut[1]:cut[2]].unflatten(1, (h, dqk)),
            z[:, cut[2]:].unflatten(1, (h, dqk)))


def _times(gen, T):
    gaps = torch.empty(T, device="cuda", dtype=torch.float64).exponential_(1.0 / GAP_MEAN_S,
                                                                          generator=gen)
    return TIME_ORIGIN + torch.cumsum(gaps.floor().long(), 0)


def _of_rows(offsets, T):
    """(user, index within the user) of each of T packed rows."""
    t = torch.arange(T, device=offsets.device)
    user = torch.searchsorted(offsets, t, right=True) - 1
    return user, t - offsets[user]


def _pages(gen, case, cap):
    """An empty cache for users of cap[b] tokens, its pages in random order and
    what is unused filled with what an earlier user left."""
    page, h = case["page"], case["heads"]
    need = [-(-n // page) for n in cap]
    pool = sum(need) + 2
    order = torch.randperm(pool, generator=gen, device="cuda").int()
    table = torch.full((case["batch"], max(1, max(need)) + 1), -1, dtype=torch.int32,
                       device="cuda")
    user, index = _of_rows(_offsets(need), sum(need))
    table[user, index] = order[:sum(need)]
    t = TYPES[case["cache"]]

    def fill(*shape):
        x = torch.randn((pool, h) + shape, generator=gen, device="cuda")
        return (x * 40).round().to(t) if t == torch.int8 else x.to(t)
    quantised = case["cache"] != "bf16"

    def scales():
        return torch.rand((pool, h, page), generator=gen, device="cuda") if quantised else None
    return {"k": fill(page, case["d_qk"]), "v": fill(case["d_v"], page),
            "timestamps": torch.full((pool, page), TIME_ORIGIN, dtype=torch.int64, device="cuda"),
            "page_table": table, "lengths": torch.tensor(cap, dtype=torch.int64, device="cuda"),
            "k_scale": scales(), "v_scale": scales()}


def _inputs(case, seed):
    """Everything that a pass starts from, the cache's contents as rows."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    h, dqk, dv = case["heads"], case["d_qk"], case["d_v"]
    s = {"case": case, "gen": gen}
    if case["op"] in ("rotary", "step"):
        s["inv_freq"] = _frequencies(case)
    if case["op"] in ("rotary", "cache"):
        lengths = _lengths(case)
        T = sum(lengths)
        s |= {"lengths": lengths, "T": T, "offsets": _offsets(lengths)}
        s["v"], s["q"], s["k"] = _fused(gen, T, h, dqk, dv, TYPES[case["dtype"]])
        if case["op"] == "cache":
            starts = _starts(case)
            s |= {"starts": torch.tensor(starts, dtype=torch.int64, device="cuda"),
                  "ends": [a + n for a, n in zip(starts, lengths)], "timestamps": _times(gen, T)}
        else:
            s["positions"] = None
            if case["far"]:
                s["positions"] = torch.randint(0, case["far"] + 1, (T,), generator=gen,
                                               device="cuda")
            if case["way"] == "bwd":
                s["q"] = torch.randn((T, h, dqk), generator=gen, device="cuda").to(s["q"].dtype)
                s["k"] = torch.randn((T, h, dqk), generator=gen, device="cuda").to(s["k"].dtype)
        return s
    hist, trees = _lengths(case), _trees(case)
    nodes = [n for n, _ in trees]
    T, M = sum(nodes), sum(hist)
    s |= {"hist": hist, "nodes": nodes, "T": T, "offsets": _offsets(nodes),
          "max_draft": max(nodes)}
    s["v"], s["q"], s["k"] = _fused(gen, T, h, dqk, dv, torch.bfloat16)
    s["hist_offsets"] = _offsets(hist)
    s["hist_v"], _, s["hist_k"] = _fused(gen, M, h, dqk, dv, torch.bfloat16)
    s["hist_time"] = _times(gen, M)
    depth = torch.tensor([d for _, par in trees for d in _depths(par)], device="cuda")
    s["timestamps"] = int(s["hist_time"][-1] if M else TIME_ORIGIN) + 30 * (1 + depth)
    s["parents"] = None
    if case["shape"] != "flat":
        s["parents"] = torch.tensor([p for _, par in trees for p in par], dtype=torch.int64,
                                    device="cuda")
    s["rab_pos"] = RAB_STD * torch.randn(2 * case["max_len"] - 1, generator=gen, device="cuda")
    s["rab_time"] = RAB_STD * torch.randn(TIME_BUCKETS, generator=gen, device="cuda")
    s["ends"] = hist
    if case["op"] == "step":
        acc = _accepted(case)
        A = sum(acc)
        s |= {"acc_offsets": _offsets(acc), "acc": acc,
              "starts": torch.tensor(hist, dtype=torch.int64, device="cuda"),
              "ends": [m + a for m, a in zip(hist, acc)]}
        s["acc_v"], _, s["acc_k"] = _fused(gen, A, h, dqk, dv, torch.bfloat16)
        user, index = _of_rows(s["acc_offsets"], A)
        s["acc_time"] = (s["hist_time"][-1] if M else TIME_ORIGIN) + index
    return s


def prepare(case, seed):
    """The tensors in hand before the call: rows, offsets and the cache."""
    s = _inputs(case, seed)
    if case["op"] == "rotary":
        return s
    s["cache"] = _pages(s["gen"], case, s["ends"])
    if case["op"] == "cache":
        if not case["write"]:
            _store(s["cache"], s["k"], s["v"], s["timestamps"], s["offsets"], s["starts"])
        return s
    zero = torch.zeros(case["batch"], dtype=torch.int64, device="cuda")
    _store(s["cache"], s["hist_k"], s["hist_v"], s["hist_time"], s["hist_offsets"], zero)
    for name in ("hist_k", "hist_v", "hist_time"):  # the cache holds them now
        del s[name]
    return s


# ------------------------------------------------------------- plain forms

def _positions(offsets, T):
    return _of_rows(offsets, T)[1]


def _rotate(x, positions, inv_freq, interleaved, back):
    """The first 2 len(inv_freq) features of each head turned in pairs."""
    half = inv_freq.numel()
    angle = positions.double()[:, None] * inv_freq[None]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    sin = -sin if back else sin
    y = x.float()
    r, rest = y[..., :2 * half], y[..., 2 * half:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :half], r[..., half:])
    a, b = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((r, rest), -1).to(x.dtype)


def _quantise(x, t):
    """Codes and scales of rows x [..., d]: the scale of an int8 row is its
    largest magnitude / 127, that of an 8-bit floating one the smallest power
    of two with which it stays within 448."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    if t == torch.int8:
        scale = torch.where(top > 0, top / 127, torch.ones_like(top))
        codes = (x.double() / scale.double()).round()
        return codes.to(torch.int8), scale[..., 0]
    mantissa, exponent = torch.frexp(torch.where(top > 0, top, torch.full_like(top, 448.0)))
    exponent = exponent - 9 + (mantissa > 0.875).int()  # 448 = 0.875 * 2^9
    scale = torch.ldexp(torch.ones_like(top), exponent)
    return torch.ldexp(x, -exponent).to(torch.float8_e4m3fn), scale[..., 0]


def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _places(cache, offsets, starts, T):
    """(page, place within it) of each of T packed rows."""
    page = cache["timestamps"].shape[1]
    user, index = _of_rows(offsets, T)
    at = starts[user] + index
    return cache["page_table"][user, at // page].long(), at % page


def _store(cache, k, v, timestamps, offsets, starts):
    page, place = _places(cache, offsets, starts, k.shape[0])
    kc, vc = k, v
    if cache["k_scale"] is not None:
        kc, ks = _quantise(k, cache["k"].dtype)
        vc, vs = _quantise(v, cache["v"].dtype)
        cache["k_scale"][page, :, place] = ks
        cache["v_scale"][page, :, place] = vs
    _bytes(cache["k"])[page, :, place] = _bytes(kc.to(cache["k"].dtype))
    _bytes(cache["v"])[page, :, :, place] = _bytes(vc.to(cache["v"].dtype))
    cache["timestamps"][page, place] = timestamps


def _load(cache, offsets, starts, T, dtype):
    page, place = _places(cache, offsets, starts, T)
    k = _bytes(cache["k"])[page, :, place].view(cache["k"].dtype).float()
    v = _bytes(cache["v"])[page, :, :, place].view(cache["v"].dtype).float()
    if cache["k_scale"] is not None:
        k = k * cache["k_scale"][page, :, place][..., None]
        v = v * cache["v_scale"][page, :, place][..., None]
    return k.to(dtype), v.to(dtype), cache["timestamps"][page, place]


def _bucket(dt):
    """min(B_t - 1, floor(log2(max(|dt|, 1)))), exact below 2^53."""
    e = torch.frexp(dt.abs().clamp_min(1).double()).exponent.long() - 1
    return e.clamp_max(TIME_BUCKETS - 1)


def _padded(x, offsets, width):
    """Packed rows [T, ...] as [users, width, ...], zeros behind each user's."""
    user, index = _of_rows(offsets, x.shape[0])
    out = x.new_zeros((offsets.numel() - 1, width) + tuple(x.shape[1:]))
    out[user, index] = x
    return out


def _ancestors(s, width):
    """[users, width, width]: 1 where a node sees another drafted one (itself
    and the nodes before it on its branch): (1 - P)^-1 = 1 + P + P^2 + ... with
    P the matrix of parents."""
    B = len(s["nodes"])
    eye = torch.eye(width, device="cuda").expand(B, width, width)
    if s["parents"] is None:
        return eye
    user, index = _of_rows(s["offsets"], s["T"])
    step = torch.zeros((B, width, width + 1), device="cuda")
    step[user, index, s["parents"] % (width + 1)] = 1.0  # -1: the last column, which is dropped
    return torch.linalg.solve_triangular(eye - step[..., :width], eye, upper=False,
                                         unitriangular=True)


def _tree_positions(s):
    """Position of each node: the cached tokens, then its depth."""
    user, index = _of_rows(s["offsets"], s["T"])
    depth = _ancestors(s, s["max_draft"]).sum(-1).round().long() - 1
    return s["cache"]["lengths"][user] + depth[user, index]


def _silu(x):
    return x / (1.0 + torch.exp(-x))


def _attend(s, q, k, v):
    """The tree attention on padded batches, in fp32."""
    N, cache, width = s["case"]["max_len"], s["cache"], s["max_draft"]
    cap = max(1, max(s["ends"]))
    page = cache["timestamps"].shape[1]
    user, index = _of_rows(s["offsets"], s["T"])
    pages = cache["page_table"][:, :-(-cap // page)].long().clamp_min(0)
    at = torch.arange(cap, device="cuda")

    def rows(x, scale, transposed):
        y = _bytes(x)[pages].view(x.dtype).float()      # [users, pages, h, page, d]
        y = y.transpose(3, 4) if transposed else y
        if scale is not None:
            y = y * scale[pages][..., None]
        return y.transpose(1, 2).flatten(2, 3)[:, :, :cap]
    kept = at[None] < cache["lengths"][:, None]         # [users, cap]
    kc = rows(cache["k"], cache["k_scale"], False)
    vc = rows(cache["v"], cache["v_scale"], True) * kept[:, None, :, None]
    seen = _ancestors(s, width) > 0.5
    depth = seen.sum(-1) - 1
    where = cache["lengths"][:, None] + depth           # [users, width]
    tq = _padded(s["timestamps"], s["offsets"], width)
    tc = cache["timestamps"][pages].flatten(1)[:, :cap]
    qp, kp, vp = (_padded(x.float(), s["offsets"], width).transpose(1, 2) for x in (q, k, v))

    def bias(key_pos, key_time):
        place = (N - 1) + key_pos[:, None, :] - where[:, :, None]
        return (s["rab_pos"][place.clamp(0, 2 * N - 2)]
                + s["rab_time"][_bucket(tq[:, :, None] - key_time[:, None, :])])

    def part(keys, values, b, mask):
        p = _silu(torch.matmul(qp, keys.transpose(2, 3)) + b[:, None])
        return torch.matmul(torch.where(mask[:, None], p, torch.zeros_like(p)), values)
    out = part(kc, vc, bias(at[None].expand_as(kept), tc), kept[:, None].expand(-1, width, -1))
    out = (out + part(kp, vp, bias(where, tq), seen)) / N
    return out.transpose(1, 2)[user, index].to(q.dtype)


def _given(s, q, k, out):
    """What a pass over a tree gives; a step has rotated rows and a cache with
    the accepted tokens too."""
    if s["case"]["op"] == "step":
        return {"out": out, "q": q, "k": k, "cache": s["cache"]}
    return out


def _run_plain(s):
    case = s["case"]
    if case["op"] == "rotary":
        at = s["positions"] if s["positions"] is not None else _positions(s["offsets"], s["T"])
        back = case["way"] == "bwd"
        return [_rotate(x, at, s["inv_freq"], case["interleaved"], back)
                for x in (s["q"], s["k"])]
    if case["op"] == "cache":
        if case["write"]:
            _store(s["cache"], s["k"], s["v"], s["timestamps"], s["offsets"], s["starts"])
        return list(_load(s["cache"], s["offsets"], s["starts"], s["T"], TYPES[case["dtype"]]))
    q, k = s["q"], s["k"]
    if case["op"] == "step":
        _store(s["cache"], s["acc_k"], s["acc_v"], s["acc_time"], s["acc_offsets"], s["starts"])
        at = _tree_positions(s)
        q, k = (_rotate(x, at, s["inv_freq"], case["interleaved"], False) for x in (q, k))
    return _given(s, q, k, _attend(s, q, k, s["v"]))


def run(state):
    """One pass: the plain form, or with `own` the library's calls."""
    if own:
        return _run_own(state)
    return _run_plain(state)


def _run_own(s):
    from paper_2402_17152_amd import hstu
    case = s["case"]
    if case["op"] == "rotary":
        call = hstu.hstu_rotary_bwd if case["way"] == "bwd" else hstu.hstu_rotary_fwd
        return list(call(s["q"], s["k"], s["inv_freq"], seq_offsets=s["offsets"],
                         positions=s["positions"], interleaved=case["interleaved"]))
    cache = hstu.PagedCache(**s["cache"])
    if case["op"] == "cache":
        if case["write"]:
            hstu.hstu_cache_write(s["k"], s["v"], s["timestamps"], s["offsets"], cache,
                                  starts=s["starts"])
        return list(hstu.hstu_cache_read(cache, s["offsets"], s["T"], starts=s["starts"],
                                         dtype=s["k"].dtype))
    q, k = s["q"], s["k"]
    if case["op"] == "step":
        hstu.hstu_cache_write(s["acc_k"], s["acc_v"], s["acc_time"], s["acc_offsets"], cache,
                              starts=s["starts"])
        at = hstu.hstu_tree_positions(s["parents"], s["offsets"], cache.lengths, s["T"],
                                      s["max_draft"])
        q, k = hstu.hstu_rotary_fwd(q, k, s["inv_freq"], positions=at,
                                    interleaved=case["interleaved"])
    out = hstu.hstu_attn_fwd_tree(q, k, s["v"], s["offsets"], s["timestamps"], cache,
                                  s["rab_pos"], s["rab_time"], case["max_len"], s["max_draft"],
                                  parents=s["parents"])
    return _given(s, q, k, out)


# ------------------------------------------- the definitions, in 64 bits

def _exact_rotate(x, positions, inv_freq, interleaved, back):
    turn = torch.exp(1j * (positions.double().outer(inv_freq)))[:, None]
    turn = turn.conj() if back else turn
    x = x.double()
    n = inv_freq.numel()
    out = x.clone()
    if interleaved:
        z = torch.view_as_complex(x[..., :2 * n].reshape(x.shape[:-1] + (n, 2)).contiguous())
        out[..., :2 * n] = torch.view_as_real(z * turn).reshape(x.shape[:-1] + (2 * n,))
    else:
        z = torch.complex(x[..., :n].contiguous(), x[..., n:2 * n].contiguous()) * turn
        out[..., :n], out[..., n:2 * n] = z.real, z.imag
    return out


def _exact_held(x, kind):
    """What a cache of this kind holds of rows x."""
    x = x.double()
    if kind == "bf16":
        return x.bfloat16().double()
    big = x.abs().max(dim=-1, keepdim=True).values
    if kind == "int8":
        unit = torch.where(big > 0, (big / 127).float().double(), 1.0)
        return torch.round(x / unit) * unit
    unit = torch.exp2(torch.ceil(torch.log2(torch.where(big > 0, big, 448.0) / 448.0)))
    unit = torch.where(big > 448.0 * unit, 2 * unit, unit)
    unit = torch.where(big <= 224.0 * unit, unit / 2, unit)
    y = x / unit
    # 3 bits behind the leading one; the smallest normal number is 2^-6
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step * unit


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "rotary":
        at = s["positions"]
        if at is None:
            at = torch.cat([torch.arange(n, device="cuda") for n in s["lengths"]])
        return [_exact_rotate(x, at, s["inv_freq"], case["interleaved"], case["way"] == "bwd")
                for x in (s["q"], s["k"])]
    if case["op"] == "cache":
        return [_exact_held(s["k"], case["cache"]), _exact_held(s["v"], case["cache"]),
                s["timestamps"]]
    hk, hv = (_exact_held(s["hist_" + n], case["cache"]) for n in "kv")
    ht = s["hist_time"]
    trees = _trees(case)
    q, k, v = (s[n].double() for n in "qkv")
    N = case["max_len"]
    pos_tab, time_tab = s["rab_pos"].double(), s["rab_time"].double()
    out, turned = torch.zeros_like(v), [torch.zeros_like(q), torch.zeros_like(k)]
    o = h0 = a0 = 0
    for b, (n, par) in enumerate(trees):
        m = s["hist"][b]
        ck, cv, ct = hk[h0:h0 + m], hv[h0:h0 + m], ht[h0:h0 + m]
        h0 += m
        if case["op"] == "step":
            a = s["acc"][b]
            ck = torch.cat((ck, _exact_held(s["acc_k"][a0:a0 + a], case["cache"])))
            cv = torch.cat((cv, _exact_held(s["acc_v"][a0:a0 + a], case["cache"])))
            ct = torch.cat((ct, s["acc_time"][a0:a0 + a]))
            a0 += a
            m += a
        line = [[i] for i in range(n)]
        for i, p in enumerate(par):
            if p >= 0:
                line[i] = line[p] + [i]
        at = torch.tensor([m + len(x) - 1 for x in line], device="cuda")
        see = torch.zeros((n, m + n), dtype=torch.bool)
        see[:, :m] = True
        for i, x in enumerate(line):
            see[i, [m + j for j in x]] = True
        see = see.cuda()
        bq, bk = q[o:o + n], k[o:o + n]
        if case["op"] == "step":  # the rotated rows are held in bf16
            bq, bk = (_exact_rotate(x, at, s["inv_freq"], case["interleaved"], False)
                      for x in (bq, bk))
            turned[0][o:o + n], turned[1][o:o + n] = bq, bk
            bq, bk = bq.bfloat16().double(), bk.bfloat16().double()
        keys, vals = torch.cat((ck, bk)), torch.cat((cv, v[o:o + n]))
        places = torch.cat((torch.arange(m, device="cuda"), at))
        stamps = torch.cat((ct, s["timestamps"][o:o + n]))
        gap = (s["timestamps"][o:o + n, None] - stamps[None]).abs().clamp_min(1)
        far = torch.floor(torch.log2(gap.double())).long().clamp_max(TIME_BUCKETS - 1)
        far -= (gap < (torch.ones_like(gap) << far)).long()
        far += (gap >= (torch.ones_like(gap) << (far + 1))).long()
        bias = pos_tab[(N - 1 + places[None] - at[:, None]).clamp(0, 2 * N - 2)] + time_tab[far]
        for a in range(case["heads"]):
            x = bq[:, a] @ keys[:, a].T + bias
            out[o:o + n, a] = ((x * torch.sigmoid(x)) * see) @ vals[:, a] / N
        o += n
    if case["op"] == "step":
        return {"out": out, "q": turned[0], "k": turned[1], "cache": None}
    return out
