"""Operators on a policy's logits against the fp64 oracle (oracle/logits.py).

Tolerances. d = c (x - m) carries three fp32 roundings and 2^d two ulp, so a
probability is off by at most 4e-7 + 2e-7 |ln p| relative; a sum of n terms adds up to
about 4 sqrt(n) 2^-25 relative (n: terms of one thread, a few thousand at most), under
7e-6. With both rounded up: ln p and LSE within 1e-5 + 2e-6 |value|, H (a sum of
terms |ln p| times larger) within 3e-5 + 2e-6 H, gradients within (1e-5 + 4e-7 |ln p|)
of the terms they are made of, plus half an ulp of the type they are stored in.
Probabilities below 2^-126 are flushed to 0, as treepo.h says.
"""
import numpy as np
import pytest
import torch

import oracle.logits as L
import paper_2508_17445_gb300 as tp
from test_gpu_parity import _built  # noqa: F401

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# half an ulp: relative, and (fp16) of the denormals
HALF_ULP = {d: (torch.finfo(t).eps / 2, 2.0 ** -25 if d == "f16" else 0.0) for d, t in TYPES.items()}
CANARY = 3.0
TINY = 2.0 ** -126 * 1e5  # probabilities below 2^-126 are 0: the whole of one, not 1e-5 of it, may be missing


def rows_like(n, v, dtype, gap=0, shift=0, fill=CANARY):
    """[n][v] inside rows of v + gap elements, starting `shift` elements into the buffer; the buffer too."""
    buf = torch.full((shift + n * (v + gap) + 16,), fill, dtype=TYPES[dtype], device=DEV)
    return buf[shift:shift + n * (v + gap)].view(n, v + gap)[:, :v], buf


def make(n, v, dtype="bf16", gap=0, shift=0, seed=0, spread=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed * 1000 + n + v)
    x, _ = rows_like(n, v, dtype, gap, shift)
    y = torch.randn((n, v), generator=g, device=DEV) * spread
    y.scatter_add_(1, torch.randint(0, v, (n, 3), generator=g, device=DEV), 8 * torch.rand((n, 3), generator=g, device=DEV))
    x.copy_(y)
    tok = torch.randint(0, v, (n,), generator=g, device=DEV).int()
    return x, tok, g


def f64(t):
    return t.detach().double().cpu().numpy()


def near(got, want, atol, rtol, what):
    got, want = f64(got), np.asarray(want, np.float64)
    with np.errstate(over="ignore"):
        want = np.where(np.isinf(want.astype(np.float32)), want.astype(np.float32), want)  # as fp32 holds it
    assert (np.isnan(got) == np.isnan(want)).all(), what
    inf = np.isinf(want)
    assert (got[inf] == want[inf]).all(), what
    ok = ~np.isnan(want) & ~inf
    d = np.abs(got[ok] - want[ok]) - rtol * np.abs(want[ok])
    assert np.isfinite(got[ok]).all() and (d <= atol).all(), (what, d.max())


def near_grad(got, want, terms, lp, dtype, extra=0.0):
    """terms: the sum of the absolute parts of each gradient that carry a probability; lp: ln p."""
    got = f64(got)
    assert (np.isnan(got) == np.isnan(want)).all()
    rel, tiny = HALF_ULP[dtype]
    lp = np.where(np.isfinite(lp), lp, 0.0)
    lim = (1e-5 + extra + 4e-7 * np.abs(lp)) * terms * (1 + 2 * rel) + (1.01 * rel + 2e-7) * np.abs(want) + 1.01 * tiny + 1e-37
    ok = ~np.isnan(want)
    d = np.abs(got - want)
    assert (d[ok] <= lim[ok]).all(), float((d[ok] / lim[ok]).max())


def check_logprobs(x, tok, k=0, temperature=1.0):
    n, v = x.shape
    f = lambda *s: torch.full(s, 7.0, device=DEV)  # noqa: E731
    out = dict(logp=f(n) if tok is not None else None, entropy=f(n), lse=f(n))
    ids, top = (torch.full((n, k), -7, dtype=torch.int32, device=DEV), f(n, k)) if k else (None, None)
    tp.tp_token_logprobs(x, tok, out["logp"], out["entropy"], out["lse"], ids, top, temperature=temperature)
    torch.cuda.synchronize()
    want = L.token_logprobs(f64(x), None if tok is None else tok.cpu().numpy(), temperature, k)
    if tok is not None:
        near(out["logp"], want["logp"], 1e-5, 2e-6, "logp")
    near(out["entropy"], want["entropy"], 3e-5, 2e-6, "entropy")
    near(out["lse"], want["lse"], 1e-5, 2e-6, "lse")
    if k:
        assert (ids.cpu().numpy() == want["top_ids"]).all()
        near(top, want["top_logp"], 1e-5, 2e-6, "top_logp")
    return out


def row_terms(x, temperature):
    rows = [L._row(r, temperature) for r in f64(x)]
    lp, p, h = (np.stack([r[i] for r in rows]) for i in (0, 1, 2))
    return np.nan_to_num(lp, nan=0.0, neginf=0.0), np.nan_to_num(p), np.nan_to_num(h)


def check_backward(x, tok, gl, gh, dtype, temperature=1.0, dx=None, buf=None):
    n, v = x.shape
    f = lambda: torch.empty(n, device=DEV)  # noqa: E731
    lse, ent = f(), f()
    tp.tp_token_logprobs(x, tok, None, ent, lse, temperature=temperature)
    keep = f64(x)
    if dx is None:
        dx, buf = rows_like(n, v, dtype)
    mark = outside(dx, buf)
    tp.tp_token_logprobs_backward(x, tok, lse, dx, gl, gh, ent if gh is not None else None, temperature=temperature)
    torch.cuda.synchronize()
    assert (outside(dx, buf) == mark).all()
    c = lambda t: None if t is None else f64(t)  # noqa: E731
    t = None if tok is None else tok.cpu().numpy()
    want = L.token_logprobs_backward(keep, t, c(lse), c(ent), c(gl), c(gh), temperature)
    lp, p, h = row_terms(torch.from_numpy(keep), temperature)
    terms = np.maximum(p, TINY) * ((np.abs(c(gl)) if gl is not None else np.zeros(n))[:, None] +
                 ((np.abs(c(gh)) if gh is not None else np.zeros(n))[:, None] * (np.abs(lp) + h[:, None] + 1))) / temperature
    size = np.abs(np.where(np.isfinite(keep), keep, 0)) / temperature + np.abs(np.nan_to_num(c(lse), neginf=0.0, posinf=0.0))[:, None]
    near_grad(dx, want, terms, lp, dtype, extra=4e-7 * size)  # x / T - lse as stored
    return dx


def outside(dx, buf):
    """The buffer's bytes that belong to no row."""
    m = torch.ones(buf.numel(), dtype=torch.bool, device=DEV)
    off = dx.storage_offset() - buf.storage_offset()
    for i in range(dx.shape[0]):
        m[off + i * dx.stride(0): off + i * dx.stride(0) + dx.shape[1]] = False
    return buf[m].float().cpu().numpy()


def check_policy(x, tok, adv, old, w, dtype, temperature=1.0, beta=0.05, dx=None, buf=None, grad=True, lo=0.2, hi=0.28):
    n, v = x.shape
    f = lambda: torch.full((n,), 7.0, device=DEV)  # noqa: E731
    loss, logp, ent = f(), f(), f()
    keep = f64(x)
    if dx is None and grad:
        dx, buf = rows_like(n, v, dtype)
    mark = outside(dx, buf) if grad else None
    tp.tp_policy_loss(x, tok, adv, loss, dx, old, w, logp, ent, clip_low=lo, clip_high=hi, entropy_coef=beta, temperature=temperature)
    torch.cuda.synchronize()
    c = lambda t: None if t is None else f64(t)  # noqa: E731
    # clip bounds and coefficient as the call takes them (fp32)
    lo, hi, beta = (float(np.float32(z)) for z in (lo, hi, beta))
    want = L.policy_loss(keep, tok.cpu().numpy(), c(adv), c(old), c(w), lo, hi, beta, temperature)
    near(logp, want["logp"], 1e-5, 2e-6, "logp")
    near(ent, want["entropy"], 3e-5, 2e-6, "entropy")
    W = np.abs(c(w)) if w is not None else np.ones(n)
    with np.errstate(over="ignore", invalid="ignore"):
        r = np.minimum(np.exp(want["logp"] - c(old)), 1e6) if old is not None else np.ones(n)
    size = np.nan_to_num(W * (np.abs(c(adv)) * (1 + r) + abs(beta)))
    near(loss / torch.tensor(np.maximum(size, 1e-30), device=DEV), want["loss"] / np.maximum(size, 1e-30), 4e-5, 4e-5, "loss")
    if grad:
        assert (outside(dx, buf) == mark).all()
        lp, p, h = row_terms(torch.from_numpy(keep), temperature)
        g = np.nan_to_num(W * np.abs(c(adv)) * r)
        terms = (np.maximum(p, TINY) * (g[:, None] + (W * abs(beta))[:, None] * (np.abs(lp) + h[:, None] + 1))) / temperature
        # the ratio's own error scales the whole row
        near_grad(dx, want["dlogits"], terms + 4e-5 / 1e-5 * np.abs(np.nan_to_num(want["dlogits"])), lp, dtype)
    return dict(loss=loss, dlogits=dx)


def check_distill(x, ids, teacher, w, dtype, temperature=1.0, dx=None, buf=None, grad=True):
    n, v = x.shape
    loss = torch.full((n,), 7.0, device=DEV)
    keep = f64(x)
    if dx is None and grad:
        dx, buf = rows_like(n, v, dtype)
    mark = outside(dx, buf) if grad else None
    tp.tp_distill_loss(x, ids, teacher, loss, dx, w, temperature=temperature)
    torch.cuda.synchronize()
    W = f64(w) if w is not None else np.ones(n)
    want = L.distill_loss(keep, ids.cpu().numpy(), f64(teacher), W, temperature)
    far = want["loss"] > 1e30  # ln p of a logit near the type's lowest value is -inf where fp32 does not hold it
    assert (f64(loss)[far] > 1e30).all()
    want["loss"][far] = f64(loss)[far]
    near(loss, want["loss"], 4e-5 * max(1.0, np.abs(W).max()), 4e-6, "loss")  # a sum of q ln q and q ln p, each within 1e-5
    if grad:
        assert (outside(dx, buf) == mark).all()
        lp, p, _ = row_terms(torch.from_numpy(keep), temperature)
        q = np.zeros((n, v))
        for i in range(n):
            at = ids[i].cpu().numpy()
            t = f64(teacher)[i]
            some = (at >= 0) & (at < v) & np.isfinite(t)
            if some.any():
                e = np.exp((t[some] - t[some].max()) / temperature)
                np.add.at(q[i], at[some], e / e.sum())
        near_grad(dx, want["dlogits"], (np.maximum(p, TINY) + q) * np.abs(W)[:, None] / temperature, lp, dtype)
    return dict(loss=loss, dlogits=dx)


def teacher_of(x, k, g, dtype=torch.float32):
    ids = torch.stack([torch.randperm(x.shape[1], generator=g, device=DEV)[:k] for _ in range(x.shape[0])]).int()
    return ids, (2 * torch.randn(ids.shape, generator=g, device=DEV)).to(dtype)


SIZES = [1, 2, 3, 7, 8, 9, 15, 31, 33, 63, 127, 255, 257, 511, 513, 1000, 2047, 4099, 8192, 12289, 32000, 50001, 65537, 100003]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", SIZES)
def test_sizes(v, dtype):
    for n, gap, shift, t in ((1, 0, 0, 1.0), (3, 5, 3, 0.7)):
        x, tok, g = make(n, v, dtype, gap, shift)
        check_logprobs(x, tok, min(v, 20), t)
        rnd = lambda: torch.randn(n, generator=g, device=DEV)  # noqa: E731
        check_backward(x, tok, rnd(), rnd(), dtype, t, *rows_like(n, v, dtype, gap, shift))
        w = torch.rand(n, generator=g, device=DEV) + 0.5
        check_policy(x, tok, rnd(), None, w, dtype, t, dx=None)
        ids, teacher = teacher_of(x, min(v, 20), g)
        check_distill(x, ids, teacher, w, dtype, t)


# rows of logits and gradients that start at different places of a 16-byte line, and in-place gradients
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("xg,xs,dg,ds", [(0, 0, 0, 1), (0, 1, 3, 0), (7, 2, 0, 5), (1, 0, 2, 0), (8, 4, 16, 4)])
def test_layouts(dtype, xg, xs, dg, ds):
    n, v = 5, 9001
    x, tok, g = make(n, v, dtype, xg, xs)
    tok[3] = -1
    rnd = lambda: torch.randn(n, generator=g, device=DEV)  # noqa: E731
    check_backward(x, tok, rnd(), rnd(), dtype, 1.0, *rows_like(n, v, dtype, dg, ds))
    check_policy(x, tok, rnd(), None, None, dtype, 1.0, 0.05, *rows_like(n, v, dtype, dg, ds))
    ids, teacher = teacher_of(x, 64, g)
    check_distill(x, ids, teacher, None, dtype, 1.0, *rows_like(n, v, dtype, dg, ds))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [77, 9001, 131072])
def test_in_place(dtype, v):
    n = 4
    for op in ("backward", "policy", "distill"):
        x, tok, g = make(n, v, dtype, 3, 1)
        tok[1] = -1
        y, buf = rows_like(n, v, dtype, 3, 1)
        y.copy_(x)
        gl, gh = torch.randn(n, generator=g, device=DEV), torch.randn(n, generator=g, device=DEV)
        if op == "backward":
            check_backward(y, tok, gl, gh, dtype, 1.0, y, buf)
        elif op == "policy":
            check_policy(y, tok, gl, None, None, dtype, 1.0, 0.05, y, buf)
        else:
            check_distill(y, *teacher_of(y, 33, g), None, dtype, 1.0, y, buf)


@pytest.mark.parametrize("dtype", TYPES)
def test_largest_vocabulary(dtype):
    v = tp.TP_MAX_VOCAB
    x, tok, g = make(2, v, dtype, 1)
    tok[1] = v - 1
    check_logprobs(x, tok, 128)
    one = torch.ones(2, device=DEV)
    check_backward(x, tok, one, one, dtype)
    check_policy(x, tok, -one, None, None, dtype)
    ids, teacher = teacher_of(x, 512, g)
    check_distill(x, ids, teacher, None, dtype)


# ------------------------------------------------------------------ values --
def special_rows(v, dtype):
    """Rows whose masks and values are where such operators go wrong, and the row's name."""
    low = float(torch.finfo(TYPES[dtype]).min)
    base = torch.linspace(-4, 4, v, device=DEV)
    rows = {"all_masked": torch.full((v,), -np.inf, device=DEV), "one_left": torch.full((v,), -np.inf, device=DEV),
            "half_masked": base.clone(), "all_lowest": torch.full((v,), low, device=DEV), "lowest_masks": base.clone(),
            "constant": torch.full((v,), 1.5, device=DEV), "zeros_of_both_signs": torch.zeros(v, device=DEV),
            "nan": base.clone(), "inf": base.clone(), "large": base * 1000, "one_large": base.clone(), "highest": base.clone(),
            "falling": -base}
    rows["one_left"][v // 2] = 3.0
    rows["half_masked"][::2] = -np.inf
    rows["lowest_masks"][v // 3:] = low
    rows["zeros_of_both_signs"][::3] = -0.0
    rows["nan"][v - 1] = np.nan
    rows["inf"][v // 2] = np.inf
    rows["one_large"][0] = 60000.0
    rows["highest"][v // 2] = float(torch.finfo(TYPES[dtype]).max)
    return torch.stack(list(rows.values())).to(TYPES[dtype]), list(rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [5, 40, 1001, 32000, 131072])
@pytest.mark.parametrize("temperature", [1.0, 0.5])
def test_special_rows(dtype, v, temperature):
    x, names = special_rows(v, dtype)
    n = len(names)
    g = torch.Generator(device=DEV).manual_seed(1)
    for at in (0, v // 2, v - 1):
        tok = torch.full((n,), at, dtype=torch.int32, device=DEV)
        if temperature == 1.0:  # (x / T of the type's extremes leaves fp32)
            check_logprobs(x, tok, min(v, 20), temperature)
        a = torch.randn(n, generator=g, device=DEV)
        # lse in fp32 does not hold ln V beside the type's extremes: those rows are left to the calls that keep the parts
        some = [i for i, r in enumerate(names) if r not in ("all_lowest", "highest") and (temperature == 1.0 or r != "one_large")]
        check_backward(x[some].contiguous(), tok[some], a[some], a[some], dtype, temperature)
        check_policy(x, tok, a, None, None, dtype, temperature)
        check_policy(x, tok, a, a - 5, None, dtype, temperature)
        ids, teacher = teacher_of(x, min(v, 5), g)
        check_distill(x, ids, teacher, None, dtype, temperature)


# the largest logits beside one another, where few threads meet them; rows in which nearly all are alternatives
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,v", [(6, 130), (6, 1000), (5000, 300), (6, 9001), (6, 40009), (6, 131072)])
def test_alternatives_in_one_place(dtype, n, v):
    x, tok, _ = make(n, v, dtype, 1)
    for i, (at, wide) in enumerate([(0, 40), (v // 2, 200), (v - 100, 100), (v // 3, v // 3)]):
        x[i, max(at, 0):at + wide] += 25
    x[4, 60:] = -np.inf
    for k in (1, 24, 25, 65, 128):
        check_logprobs(x, tok, k)


# either side of the row sizes and row counts at which another kernel takes over, rows at any place
@pytest.mark.parametrize("n,v,dtype", [(610, 24570, "bf16"), (610, 24577, "f16"), (600, 16385, "bf16"), (303, 10241, "f16"), (305, 10240, "bf16"),
                                       (304, 8193, "f32"), (20, 5120, "f32"), (20, 5121, "f32")])
def test_kernel_boundaries(n, v, dtype):
    x, tok, g = make(n, v, dtype, 3, 1)
    tok[::7] = -1
    a = torch.randn(n, generator=g, device=DEV)
    check_logprobs(x, tok)
    check_logprobs(x, tok, 20)
    check_policy(x, tok, a, None, None, dtype, 0.8)
    ids, teacher = teacher_of(x, 20, g)
    check_distill(x, ids, teacher, None, dtype, 0.8, *rows_like(n, v, dtype, 1, 3))


# masks by finite values that stay finite as x / T, with coefficients that take their product past fp32
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,v", [(3, 700), (2100, 300), (3, 9001), (3, 40000)])
def test_far_masks_and_large_coefficients(dtype, n, v):
    x, tok, g = make(n, v, dtype)
    a = torch.randn(n, generator=g, device=DEV)
    for mask in (-3e38, -1e30, -np.inf):
        x[:, v // 2:] = mask
        x[:, v // 3] = -3e38
        tok[0], tok[1] = v // 2 - 1, v - 1
        check_policy(x, tok, a, None, None, dtype, 2.0, beta=8.0)
        check_policy(x, tok, a, None, torch.full((n,), 1e4, device=DEV), dtype, 2.0)
        check_backward(x, tok, a, 1e9 * (a.abs() + 1), dtype, 2.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_out_of_range_and_padding(dtype):
    v = 5000
    x, _, g = make(7, v, dtype)
    tok = torch.tensor([-1, 0, v - 1, v, 2 ** 31 - 1, -2 ** 31, 17], dtype=torch.int32, device=DEV)
    x[5] = float("nan")  # a padding row is not looked at
    check_logprobs(x, tok, 3)
    a = torch.randn(7, generator=g, device=DEV)
    check_backward(x, tok, a, a, dtype)
    check_backward(x, tok, a, None, dtype)
    check_policy(x, tok, a, None, None, dtype)


def test_logprobs_without_tokens_and_parts():
    x, tok, g = make(4, 3001)
    check_logprobs(x, None, 5)
    gh = torch.randn(4, generator=g, device=DEV)
    check_backward(x, None, None, gh, "bf16")
    check_backward(x, tok, gh, None, "bf16")
    for name in ("logp", "entropy", "lse"):
        out = torch.full((4,), 7.0, device=DEV)
        tp.tp_token_logprobs(x, tok, **{name: out})
        near(out, L.token_logprobs(f64(x), tok.cpu().numpy())[name], 3e-5, 2e-6, name)
    tp.tp_token_logprobs(x, tok)  # nothing asked for


# -------------------------------------------------------------- alternatives --
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [1, 2, 31, 64, 127, 128])
@pytest.mark.parametrize("v", [128, 1000, 40009, 131072])
def test_alternatives(dtype, k, v):
    x, tok, _ = make(3, v, dtype, 1)
    check_logprobs(x, tok, k)


# few distinct values, rising, falling, periodic: many equal logits, or all of the largest in one place
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v", [200, 4096, 33333, 131072])
def test_alternatives_among_equals(dtype, v):
    at = torch.arange(v, device=DEV)
    few = torch.randint(0, 3, (v,), generator=torch.Generator(device=DEV).manual_seed(v), device=DEV)
    block = torch.where((at >= v // 2) & (at < v // 2 + 150), 50.0, 0.0) + (at % 7) * 0.25
    rows = [few.float(), -(at.float() / v * 8), at.float() / v * 8, (at % 97).float() / 16, block, torch.zeros(v, device=DEV),
            torch.where(at % 512 == 3, 4.0 + at / v, -1.0), torch.where(at < 10, 1.0, -torch.inf)]
    x = torch.stack(rows).to(TYPES[dtype])
    for k in (1, 20, 128):
        check_logprobs(x, torch.zeros(len(rows), dtype=torch.int32, device=DEV), k)


# ------------------------------------------------------------------- losses --
@pytest.mark.parametrize("dtype", TYPES)
def test_policy_clips(dtype):
    n, v = 64, 2000
    x, tok, g = make(n, v, dtype)
    lp = torch.empty(n, device=DEV)
    tp.tp_token_logprobs(x, tok, lp)
    ratio = torch.linspace(0.5, 1.6, n, device=DEV)  # (none within 1e-3 of 0.8 or 1.28)
    assert min((ratio - e).abs().min() for e in (0.8, 1.28)) > 1e-3
    for a in (1.0, -1.0, 0.0):
        adv = torch.full((n,), a, device=DEV)
        r = check_policy(x, tok, adv, lp - ratio.log(), torch.rand(n, generator=g, device=DEV), dtype, beta=0.0)
        if a:
            held = (ratio > 1.28) if a > 0 else (ratio < 0.8)
            assert ((r["dlogits"] == 0).all(1) == held).all()
    check_policy(x, tok, torch.ones(n, device=DEV), lp, None, dtype, grad=False)
    # a ratio that overflows: the clip holds it for A > 0
    check_policy(x, tok, torch.ones(n, device=DEV), lp - 200, None, dtype, beta=0.0)
    check_policy(x, tok, torch.zeros(n, device=DEV), lp - 200, None, dtype, beta=0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [1, 3, 64, 300, 512])
def test_distill_lists(dtype, k):
    n, v = 9, 7001
    x, _, g = make(n, v, dtype, 1)
    for td in TYPES.values():
        ids, t = teacher_of(x, k, g, td)
        ids[1] = -1                       # padding
        t[2] = -np.inf                    # padding too
        ids[3, k // 2:] = -1              # a shorter list
        t[4, : k // 2] = -np.inf          # entries without a share
        ids[5] = ids[5, 0].clone()        # one id throughout
        ids[6, 0] = v                     # out of range: NaN
        t[7, k - 1] = np.nan
        ids[8] = torch.arange(k, device=DEV).int()  # neighbours
        check_distill(x, ids, t, torch.rand(n, generator=g, device=DEV) + 0.5, dtype, 2.0)
        check_distill(x, ids, t, None, dtype, grad=False)


def test_distill_of_ones_own_alternatives():
    """All of a short vocabulary listed by tp_token_logprobs: the teacher agrees with itself, loss and gradient vanish."""
    x, tok, _ = make(6, 100, "f32")
    ids, top = torch.empty((6, 100), dtype=torch.int32, device=DEV), torch.empty((6, 100), device=DEV)
    tp.tp_token_logprobs(x, tok, top_ids=ids, top_logp=top)
    loss, dx = torch.empty(6, device=DEV), torch.empty_like(x)
    tp.tp_distill_loss(x, ids, top, loss, dx)
    assert loss.abs().max() < 1e-5 and dx.abs().max() < 1e-6


def test_gradients_against_differences_of_the_losses():
    """Central differences of the kernels' own fp32 losses, h = 2^-4: rounding 4e-6 / h below 1e-4, h^2 / 6 of the third
    derivative (at most about 1 for these sizes) below 1e-3."""
    n, v, h = 1, 50, 2.0 ** -4
    x, tok, g = make(n, v, "f32", spread=1.0)
    step = torch.cat([x + h * torch.eye(v, device=DEV), x - h * torch.eye(v, device=DEV)])
    m = 2 * v
    rep = lambda t: t.expand(m, *t.shape[1:]).contiguous()  # noqa: E731
    slope = lambda l: (l[:v] - l[v:]) / (2 * h)  # noqa: E731
    adv = torch.tensor([0.7], device=DEV)
    lp = torch.empty(1, device=DEV)
    tp.tp_token_logprobs(x, tok, lp, temperature=1.5)
    old = lp - 0.05
    loss, dx, many = torch.empty(1, device=DEV), torch.empty_like(x), torch.empty(m, device=DEV)
    kw = dict(clip_low=0.9, clip_high=3.0, entropy_coef=0.3, temperature=1.5)
    tp.tp_policy_loss(x, tok, adv, loss, dx, old, **kw)
    tp.tp_policy_loss(step, rep(tok), rep(adv), many, None, rep(old), **kw)
    assert (slope(many) - dx[0]).abs().max() < 2e-3
    ids, t = teacher_of(x, 8, g)
    tp.tp_distill_loss(x, ids, t, loss, dx, temperature=1.5)
    tp.tp_distill_loss(step, rep(ids), rep(t), many, temperature=1.5)
    assert (slope(many) - dx[0]).abs().max() < 2e-3
    ent, lse, ones = torch.empty(m, device=DEV), torch.empty(1, device=DEV), torch.ones(1, device=DEV)
    e1 = torch.empty(1, device=DEV)
    tp.tp_token_logprobs(x, tok, lp, e1, lse)
    tp.tp_token_logprobs(step, rep(tok), many, ent)
    tp.tp_token_logprobs_backward(x, tok, lse, dx, ones, -2 * ones, e1)
    assert (slope(many - 2 * ent) - dx[0]).abs().max() < 4e-3


# ------------------------------------------------------------ calls, streams --
def test_another_stream_graph_and_repeats():
    n, v = 37, 50001
    x, tok, g = make(n, v)
    a = torch.randn(n, generator=g, device=DEV)
    ids, teacher = teacher_of(x, 64, g)

    def once(**kw):
        o = {s: torch.empty(n, device=DEV) for s in ("logp", "entropy", "lse", "loss", "kl")}
        o["ids"], o["top"] = torch.empty((n, 50), dtype=torch.int32, device=DEV), torch.empty((n, 50), device=DEV)
        o["dp"], o["dk"], o["db"] = (torch.empty_like(x) for _ in range(3))

        def go():
            tp.tp_token_logprobs(x, tok, o["logp"], o["entropy"], o["lse"], o["ids"], o["top"], **kw)
            tp.tp_token_logprobs_backward(x, tok, o["lse"], o["db"], a, a, o["entropy"], **kw)
            tp.tp_policy_loss(x, tok, a, o["loss"], o["dp"], o["logp"], entropy_coef=0.1, **kw)
            tp.tp_distill_loss(x, ids, teacher, o["kl"], o["dk"], **kw)
        return o, go

    first, go = once()
    go()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        second, go = once()  # torch's current stream
        go()
    third, go3 = once(stream=side)
    torch.cuda.synchronize()
    go3()
    graph = torch.cuda.CUDAGraph()
    fourth, go4 = once()
    with torch.cuda.graph(graph):
        go4()
    graph.replay()
    torch.cuda.synchronize()
    for name, want in first.items():
        for got in (second[name], third[name], fourth[name]):
            assert torch.equal(got, want), name


def test_rows_past_2_31_elements():
    """Offsets that pass 32 bits: the last rows of 4.5 GB of logits, gradient in place."""
    n, v = 17500, 131072
    x = torch.zeros((n, v), dtype=torch.bfloat16, device=DEV)
    last, tok3, g = make(3, v)
    x[-3:] = last
    tok = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    tok[-3:] = tok3
    adv, loss, lp = torch.ones(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    tp.tp_token_logprobs(x, tok, lp)
    tp.tp_policy_loss(x, tok, adv, loss, x)
    want = L.policy_loss(f64(last), tok3.cpu().numpy(), [1.0, 1.0, 1.0])
    near(lp[-3:], want["logp"], 1e-5, 2e-6, "logp")
    near(loss[-3:], want["loss"], 4e-5, 4e-5, "loss")
    lps, p, _ = row_terms(last, 1.0)
    near_grad(x[-3:], want["dlogits"], p, lps, "bf16")
    assert not loss[:-3].any() and not x[:-3].any()


def test_many_rows_of_a_small_vocabulary():
    n, v = 70001, 33
    x, tok, g = make(n, v, "f32")
    tok[::5] = -1
    check_logprobs(x, tok, 4)
    check_policy(x, tok, torch.randn(n, generator=g, device=DEV), None, None, "f32")


def test_binding_refuses():
    x, tok, _ = make(4, 100)
    one = torch.ones(4, device=DEV)
    for call in (lambda: tp.tp_token_logprobs(x, tok.long(), one), lambda: tp.tp_token_logprobs(x, tok, one.double()),
                 lambda: tp.tp_token_logprobs(x, tok, one[:3]), lambda: tp.tp_token_logprobs(x.double(), tok, one),
                 lambda: tp.tp_token_logprobs(x.t(), tok, one), lambda: tp.tp_token_logprobs(x, tok, one, top_ids=tok[:, None]),
                 lambda: tp.tp_token_logprobs(x, tok.cpu(), one),
                 lambda: tp.tp_policy_loss(x, tok, one, one.clone(), x.float()),
                 lambda: tp.tp_policy_loss(x, tok, one, one.clone(), torch.empty_like(x)[:, :50]),
                 lambda: tp.tp_distill_loss(x, tok[:, None], one[:3, None], one.clone())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(tp.TreepoError):
        tp.tp_token_logprobs(x, None, one)  # logp without tokens
    with pytest.raises(tp.TreepoError):
        tp.tp_token_logprobs(x[:1].expand(4, 100), tok, one)
    e = torch.empty(0, device=DEV)
    tp.tp_token_logprobs(x[:0], tok[:0], e, e)


# ------------------------------------------------- many rows, in 64 bits on the GPU --
def many(n, v, dtype, seed):
    """Rows in more rounds than the GPU has places for, a third of them padding, a few of the rest special."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.empty((n, v), dtype=TYPES[dtype], device=DEV)
    for a in range(0, n, 256):
        x[a:a + 256] = torch.randn((min(256, n - a), v), generator=g, device=DEV) * 2.5
    x[5, : v // 2] = -torch.inf
    x[6] = -torch.inf
    x[7, 11] = torch.nan
    x[8] = 0.5
    x[9, 100:] = -torch.inf
    tok = torch.randint(0, v, (n,), generator=g, device=DEV).int()
    tok[torch.rand(n, generator=g, device=DEV) < 0.33] = -1
    tok[:10] = torch.arange(10, device=DEV).int()
    return x, tok, g


def in_parts(x, f):
    parts = [f(x[a:a + 128].double(), slice(a, a + 128)) for a in range(0, len(x), 128)]
    return [torch.cat(p) for p in zip(*parts)]


@pytest.mark.parametrize("dtype,n,v", [("bf16", 1900, 40000), ("bf16", 1830, 33001), ("f32", 1850, 20001), ("bf16", 700, 150000),
                                       ("f16", 320, 33333)])
def test_many_rows(dtype, n, v):
    x, tok, g = many(n, v, dtype, n + v)
    live, at = tok >= 0, tok.long().clamp(min=0)[:, None]
    k = 9

    def exact(y, rows):
        y = torch.where(torch.isnan(y).any(1, keepdim=True), torch.nan, y)
        lse = torch.logsumexp(y, -1)
        lp = y - lse[:, None]
        lp = torch.where((lse == -torch.inf)[:, None], -torch.inf, lp)
        p = lp.exp()
        h = -torch.where(p > 0, p * lp, p * 0).sum(1)
        top = torch.where(torch.isnan(lse)[:, None], torch.nan, lp.topk(k, -1).values)
        return lp.gather(1, at[rows])[:, 0], h, lse, top
    logp, h, lse, top = in_parts(x, exact)
    f = lambda *s: torch.full(s, 7.0, device=DEV)  # noqa: E731
    glp, gh, gl, ids, gtop = f(n), f(n), f(n), torch.full((n, k), -7, dtype=torch.int32, device=DEV), f(n, k)
    tp.tp_token_logprobs(x, tok, glp, gh, gl, ids, gtop)
    near(glp, f64(torch.where(live, logp, 0.0)), 1e-5, 2e-6, "logp")
    near(gh, f64(torch.where(live, h, 0.0)), 3e-5, 2e-6, "entropy")
    near(gl, f64(torch.where(live, lse, 0.0)), 1e-5, 2e-6, "lse")
    near(gtop, f64(torch.where(live[:, None], top, -torch.inf)), 1e-5, 2e-6, "top_logp")
    some = ids >= 0
    assert ((ids == -1) | some).all()
    # the ids are the places of these logits, equal ones in rising order
    vals = x.gather(1, ids.long().clamp(min=0)).float()
    fine = some[:, 1:] & some[:, :-1]
    assert ((vals[:, 1:] < vals[:, :-1]) | ((vals[:, 1:] == vals[:, :-1]) & (ids[:, 1:] > ids[:, :-1])))[fine].all()
    near(torch.where(some, vals - gl[:, None], gtop), f64(gtop), 2e-5, 4e-6, "ids")

    adv, w = torch.randn(n, generator=g, device=DEV), torch.rand(n, generator=g, device=DEV) + 0.5
    tid = torch.randint(0, v, (n, 20), generator=g, device=DEV).int()
    tval = torch.randn((n, 20), generator=g, device=DEV)
    tid[~live] = -1
    beta = 0.05
    loss, kl = f(n), f(n)
    dp, dk = torch.empty_like(x), x.clone()
    tp.tp_policy_loss(x, tok, adv, loss, dp, None, w, entropy_coef=beta)
    tp.tp_distill_loss(dk, tid, tval, kl, dk, w)  # in place
    q = torch.softmax(tval.double(), -1)
    beta = float(np.float32(beta))

    def grads(y, rows):
        y = torch.where(torch.isnan(y).any(1, keepdim=True), torch.nan, y)
        empty = (y == -torch.inf).all(1, keepdim=True)
        lp = torch.where(empty, -torch.inf, y - torch.logsumexp(y, -1, keepdim=True))
        p, l = lp.exp(), live[rows, None]
        a, ww = -adv[rows].double()[:, None], w[rows].double()[:, None]
        hh = torch.where(p > 0, p * lp, p * 0)
        d = a * (torch.zeros_like(p).scatter_(1, at[rows], 1.0) - p) + beta * (hh - p * hh.sum(1, keepdim=True))
        d = torch.where(empty, 0.0, d) * ww
        t = torch.where(empty, 0.0, p.scatter_add(1, tid[rows].long().clamp(min=0), -q[rows])) * ww
        d, t = torch.where(l, d, 0.0), torch.where(l, t, 0.0)
        # half an ulp of the type, the few fp32 roundings of a row's factors, 1e-4 of a probability's share
        u, tiny = HALF_ULP[dtype]
        u += 5e-7
        size = (p * (a.abs() + beta * (lp.clamp(min=-200).abs() - hh.sum(1, keepdim=True) + 1)) * ww).nan_to_num()
        far_d = ((dp[rows].double() - d).abs() - 1.05 * u * d.abs() - 1e-4 * size - 1.01 * tiny - 1e-37)
        far_t = ((dk[rows].double() - t).abs() - 1.05 * u * t.abs() - 1e-4 * (p * ww).nan_to_num() - 1e-6 * q[rows].amax(1, keepdim=True) * ww
                 - 1.01 * tiny - 1e-37)
        ok = lambda far, got, want: (torch.isnan(got) == torch.isnan(want)).all(1) & ((far <= 0) | torch.isnan(far)).all(1)  # noqa: E731
        return ok(far_d, dp[rows], d), ok(far_t, dk[rows], t)
    okd, okt = in_parts(x, grads)
    assert okd.all(), torch.nonzero(~okd)[:5, 0].tolist()
    assert okt.all(), torch.nonzero(~okt)[:5, 0].tolist()
    want = torch.where(live, w * (-adv - beta * h), 0.0)
    near(loss[live & ~torch.isnan(want)], f64(want[live & ~torch.isnan(want)]), 1e-4, 4e-6, "loss")
    assert (loss[~live] == 0).all() and (kl[~live] == 0).all()
