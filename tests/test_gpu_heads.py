"""Norm and rotation of heads and their gradients on the GPU, against the 64-bit definition."""
import numpy as np
import pytest
import torch

from oracle import heads_ref as H
from operator_graphs import Graph, rounded
from paper_2405_16283_amd import binding as B

pytestmark = pytest.mark.gpu
EPS = 1e-5
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24

# rows, heads, head size, and what differs from: half pairs, whole heads rotated, plain frequencies, row r at position r, a norm
CASES = [
    dict(rows=1, heads=1, hd=2),
    dict(rows=1, heads=32, hd=128, pos0=100003),
    dict(rows=5, heads=3, hd=64, half=0),
    dict(rows=67, heads=2, hd=128, half=0, rotary=32),
    dict(rows=67, heads=2, hd=128, rotary=64, norm=0),
    dict(rows=33, heads=5, hd=80, rotary=20),
    dict(rows=33, heads=3, hd=96, half=0),
    dict(rows=31, heads=7, hd=96, norm=0),
    dict(rows=9, heads=3, hd=66, rotary=22),
    dict(rows=10, heads=2, hd=10, half=0, rotary=6),
    dict(rows=65, heads=2, hd=256, positions=1),
    dict(rows=64, heads=2, hd=512, half=0),
    dict(rows=3, heads=2, hd=1024, positions=1),
    dict(rows=200, heads=4, hd=64, positions=1, factor=8.0, len0=512),
    dict(rows=130, heads=8, hd=128, factor=4.0, base=500000.0, pos0=70000),
    dict(rows=100, heads=8, hd=128, factor=4.0, len0=8192, base=500000.0, half=0, positions=1),
]


def _setup(c, dtype, seed):
    rng = np.random.default_rng(seed)
    rows, hd = c["rows"], c["hd"]
    d = c["heads"] * hd
    x = rounded(rng.standard_normal((rows, d)) * np.exp(rng.standard_normal((rows, 1))), dtype)
    gain = rounded(1 + 0.2 * rng.standard_normal((1, hd)), dtype)
    dy = rounded(rng.standard_normal((rows, d)), dtype)
    pos0 = c.get("pos0", 0)
    own = rng.integers(-5, 200000, (rows, 1)) if c.get("positions") else None
    at = torch.as_tensor(pos0 + (own[:, 0] if own is not None else np.arange(rows)))
    rd = c.get("rotary", 0) or hd
    freq = H.frequencies(rd, c.get("base", 10000.0), c.get("factor", 0.0), c.get("len0", 0), 1.0, 4.0)
    par = dict(head_dim=hd, pos0=pos0, rope_base=c.get("base", 10000.0), rotary_dim=c.get("rotary", 0), rope_half=c.get("half", 1),
               positions=int(own is not None), norm=c.get("norm", 1), eps=EPS, rope_factor=c.get("factor", 0.0), rope_len0=c.get("len0", 0),
               rope_low=1.0, rope_high=4.0)
    return x, gain, dy, own, at, freq, par


def _pair_size(n, hd, freq, half):
    """|a| + |b| of the pair an element belongs to (an element that stays: its own size)."""
    a = np.abs(n).reshape(n.shape[0], -1, hd)
    s, k = a.copy(), len(freq)
    if half:
        s[..., :k] = s[..., k:2 * k] = a[..., :k] + a[..., k:2 * k]
    else:
        s[..., 0:2 * k:2] = s[..., 1:2 * k:2] = a[..., 0:2 * k:2] + a[..., 1:2 * k:2]
    return s.reshape(n.shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_forward(c, dtype):
    x, gain, _, own, at, freq, par = _setup(c, dtype, 1)
    g = Graph(dtype)
    ins = [g.inp(x)] + ([g.inp(gain)] if par["norm"] else []) + ([g.inp(own, "i32")] if own is not None else [])
    (out,) = g.run([g.op(B.TN_OP_HEAD_ROPE, ins, *x.shape, **par)])
    n = H.head_norm(torch.tensor(x), c["hd"], torch.tensor(gain), EPS) if par["norm"] else torch.tensor(x)
    ref = H.head_rotate(n, c["hd"], at, freq, bool(par["rope_half"])).numpy()
    # the norm: a sum of hd squares and a few operations; sine and cosine: a few units of 1; one rounding to storage
    tol = STEP[dtype] * np.abs(ref) + (c["hd"] / 2 + 24) * U * _pair_size(n.numpy(), c["hd"], freq, par["rope_half"])
    assert (np.abs(out - ref) <= tol).all(), np.max(np.abs(out - ref) / np.maximum(tol, 1e-30))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_backward(c, dtype):
    x, gain, dy, own, at, freq, par = _setup(c, dtype, 2)
    hd, rows = c["hd"], c["rows"]
    g = Graph(dtype)
    pos = [g.inp(own, "i32")] if own is not None else []
    if not par["norm"]:  # the gradient of a rotation is its inverse
        (out,) = g.run([g.op(B.TN_OP_HEAD_ROPE, [g.inp(dy)] + pos, *x.shape, mode=1, **par)])
        ref = H.head_rotate(torch.tensor(dy), hd, at, freq, bool(par["rope_half"]), inverse=True).numpy()
        tol = STEP[dtype] * np.abs(ref) + 24 * U * _pair_size(dy, hd, freq, par["rope_half"])
        assert (np.abs(out - ref) <= tol).all()
        return
    ins = [g.inp(dy), g.inp(x), g.inp(gain)] + pos
    dx = g.op(B.TN_OP_HEAD_ROPE_BWD, ins, *x.shape, **par)
    pieces = (rows + 31) // 32
    part = g.op(B.TN_OP_HEAD_ROPE_BWD, ins, pieces, hd, "f32", mode=1, **par)
    total = g.op(B.TN_OP_COL_SUM, [part], 1, hd, "f32")
    gx, gp, gg = g.run([dx, part, total])
    X, G = torch.tensor(x, requires_grad=True), torch.tensor(gain, requires_grad=True)
    y = H.head_rotate(H.head_norm(X, hd, G, EPS), hd, at, freq, bool(par["rope_half"]))
    rx, rg = torch.autograd.grad(y, (X, G), torch.tensor(dy))
    # element by element: u and n as in the forward pass; the mean of hd products relative to the sum of their sizes
    heads = lambda a: a.reshape(rows, -1, hd)  # noqa: E731
    r = 1 / np.sqrt((heads(x) ** 2).mean(-1, keepdims=True) + EPS)
    n, ua = np.abs(heads(x)) * r, heads(_pair_size(dy, hd, freq, par["rope_half"]))
    size = r * (ua * np.abs(gain) + n * (ua * np.abs(gain) * n).mean(-1, keepdims=True))
    tol = STEP[dtype] * np.abs(rx.numpy()) + (hd + 40) * U * size.reshape(rows, -1)
    assert (np.abs(gx - rx.numpy()) <= tol).all(), np.max(np.abs(gx - rx.numpy()) / tol)
    size = (ua * n).sum((0, 1))
    tol = (rows * c["heads"] + hd + 40) * U * size
    assert (np.abs(gg[0] - rg.numpy()[0]) <= tol).all()
    u = H.head_rotate(torch.tensor(dy), hd, at, freq, bool(par["rope_half"]), inverse=True).numpy().reshape(rows, -1, hd)
    each = (u * heads(x) * r).sum(1)
    for i in range(pieces):
        assert (np.abs(gp[i] - each[32 * i:32 * i + 32].sum(0)) <= tol).all()


def test_gradients_against_differences():
    c = CASES[3]
    x, gain, dy, own, at, freq, par = _setup(c, "f32", 3)
    g = Graph()
    ins = [g.inp(dy), g.inp(x), g.inp(gain)]
    gx, gp = g.run([g.op(B.TN_OP_HEAD_ROPE_BWD, ins, *x.shape, **par), g.op(B.TN_OP_HEAD_ROPE_BWD, ins, (c["rows"] + 31) // 32, c["hd"], "f32", mode=1, **par)])

    def loss(x, gain):
        y = H.head_rotate(H.head_norm(torch.tensor(x), c["hd"], torch.tensor(gain), EPS), c["hd"], at, freq, bool(par["rope_half"]))
        return float((y * torch.tensor(dy)).sum())

    rng, h = np.random.default_rng(4), 1e-5
    for _ in range(10):
        step = rng.standard_normal(x.shape)
        slope = (loss(x + h * step, gain) - loss(x - h * step, gain)) / (2 * h)
        assert abs(slope - (gx * step).sum()) <= 1e-5 * np.abs(gx * step).sum()  # fp32 sums of the gradient, h^2 of the difference
        step = rng.standard_normal(gain.shape)
        slope = (loss(x, gain + h * step) - loss(x, gain - h * step)) / (2 * h)
        assert abs(slope - (gp.sum(0) * step).sum()) <= 1e-5 * np.abs(gp * step).sum()


def test_heads_of_one_launch_differ_in_everything():
    """Vertices of several sizes, layouts and positions go in one launch."""
    g, outs, refs = Graph("bf16"), [], []
    for k, c in enumerate(CASES):
        x, gain, _, own, at, freq, par = _setup(c, "bf16", 10 + k)
        ins = [g.inp(x)] + ([g.inp(gain)] if par["norm"] else []) + ([g.inp(own, "i32")] if own is not None else [])
        outs.append(g.op(B.TN_OP_HEAD_ROPE, ins, *x.shape, **par))
        n = H.head_norm(torch.tensor(x), c["hd"], torch.tensor(gain), EPS) if par["norm"] else torch.tensor(x)
        refs.append((H.head_rotate(n, c["hd"], at, freq, bool(par["rope_half"])).numpy(), _pair_size(n.numpy(), c["hd"], freq, par["rope_half"])))
    for out, (ref, size) in zip(g.run(outs), refs):
        assert (np.abs(out - ref) <= 2.0 ** -8 * np.abs(ref) + 600 * U * size).all()


def test_a_row_of_zeros_and_one_that_is_not_finite():
    c = dict(rows=70, heads=2, hd=128)
    x, gain, dy, _, at, freq, par = _setup(c, "f32", 5)
    x[3] = 0
    x[5, 7] = np.inf
    x[6, 130] = np.nan
    g = Graph()
    i, j = g.inp(x), g.inp(gain)
    y, dx = g.run([g.op(B.TN_OP_HEAD_ROPE, [i, j], *x.shape, **par), g.op(B.TN_OP_HEAD_ROPE_BWD, [g.inp(dy), i, j], *x.shape, **par)])
    assert (y[3] == 0).all() and np.isfinite(dx[3]).all()
    bad = np.zeros((70, 2), bool)
    bad[5, 0] = bad[6, 1] = True  # the other head of the row, and other rows, are left alone
    for a in (y, dx):
        assert (np.isfinite(a.reshape(70, 2, 128)).all(-1) == ~bad).all()


def test_sums_of_columns():
    rng = np.random.default_rng(6)
    for shapes, cols in (([1], 1), ([5, 1, 300], 33), ([512], 128), ([3, 17], 1024)):
        g = Graph()
        parts = [rng.standard_normal((r, cols)).astype(np.float32) for r in shapes]
        (out,) = g.run([g.op(B.TN_OP_COL_SUM, [g.inp(p) for p in parts], 1, cols, "f32")])
        a = np.concatenate(parts).astype(np.float64)
        assert (np.abs(out[0] - a.sum(0)) <= len(a) * U * np.abs(a).sum(0)).all()


def test_more_heads_than_a_launch_has_wavefronts():
    c = dict(rows=300001, heads=4, hd=6)
    test_forward(c, "f32")
    test_backward(c, "f32")
