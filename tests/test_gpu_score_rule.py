"""Attention by a score rule on the GPU, forward and reverse, against the 64-bit definition; bounds count the roundings."""
import math

import numpy as np
import pytest
import torch

from oracle import heads_ref as H
from operator_graphs import Graph, rounded
from paper_2405_16283_amd import binding as B

pytestmark = pytest.mark.gpu
BIG = 2 ** 31 - 1


def _documents(rows, cuts, padding=0):
    s = np.zeros((rows, 2), np.int64)
    b = [0] + list(cuts) + [rows - padding]
    for lo, hi in zip(b, b[1:]):
        s[lo:hi] = lo, hi
    return s


def _prefix(rows, n):
    at = np.arange(rows)
    return np.stack([np.zeros(rows), np.maximum(at + 1, n)], 1)


def _window(rows, n, keys=None, first=0):
    at = np.arange(rows) + first
    return np.stack([np.maximum(at - n + 1, 0), np.full(rows, BIG)], 1)


def _holes(rows, keys, seed):
    """Any spans at all: empty ones, reversed ones, ones outside."""
    rng = np.random.default_rng(seed)
    s = np.sort(rng.integers(-20, keys + 20, (rows, 2)), 1)
    s[rng.random(rows) < 0.2] = 7, 7
    s[rng.random(rows) < 0.1] = 9, 3
    s[rng.random(rows) < 0.1] = -BIG - 1, BIG
    s[rng.random(rows) < 0.1] = keys + 1000, BIG
    return s


# rows, keys, heads, head size; differing from: tiles as large as the tensors, causal, no cap, no slopes, no spans
CASES = {
    "one": dict(rows=1, keys=1, heads=1, hd=64, cap=5.0),
    "one row": dict(rows=1, keys=333, heads=3, hd=128, causal=0, cap=20.0, slopes=1, q_pos0=332),
    "one key": dict(rows=70, keys=1, heads=2, hd=64, causal=0, cap=20.0),
    "capped": dict(rows=160, keys=160, heads=3, hd=64, cap=3.0),
    "capped far": dict(rows=130, keys=130, heads=2, hd=128, cap=0.5, std=6.0),
    "slopes": dict(rows=161, keys=161, heads=4, hd=128, slopes=1),
    "slopes both ways": dict(rows=65, keys=200, heads=2, hd=64, causal=0, slopes=1, q_pos0=90),
    "documents": dict(rows=333, keys=333, heads=2, hd=128, spans=_documents(333, [5, 70, 71, 200], 20), cap=30.0),
    "documents in tiles": dict(rows=300, keys=300, heads=4, hd=64, tile=128, spans=_documents(300, [64, 128, 129], 44), slopes=1),
    "prefix": dict(rows=270, keys=270, heads=2, hd=128, causal=0, spans=_prefix(270, 100), cap=50.0),
    "prefix in tiles": dict(rows=257, keys=257, heads=2, hd=128, tile=128, causal=0, spans=_prefix(257, 65)),
    "window": dict(rows=400, keys=400, heads=1, hd=64, spans=_window(400, 33), cap=50.0, slopes=1),
    "window of one": dict(rows=129, keys=129, heads=2, hd=128, spans=_window(129, 1)),
    "behind a cache": dict(rows=37, keys=500, heads=2, hd=128, q_pos0=463, spans=_window(37, 300, first=463), cap=10.0, tile=256),
    "cut off keys": dict(rows=90, keys=64, heads=2, hd=64, q_pos0=0, k_pos0=40, cap=10.0),
    "holes": dict(rows=200, keys=190, heads=2, hd=128, causal=0, spans=_holes(200, 190, 1)),
    "holes and all": dict(rows=191, keys=333, heads=3, hd=64, causal=1, q_pos0=100, spans=_holes(191, 333, 2), cap=7.0, slopes=1, tile=64),
    "nothing": dict(rows=66, keys=66, heads=1, hd=128, spans=np.zeros((66, 2))),
    "far positions": dict(rows=70, keys=140, heads=2, hd=64, q_pos0=2 ** 30 - 70, k_pos0=2 ** 30 - 140, slopes=1, cap=9.0,
                          spans=_window(70, 50, first=2 ** 30 - 70)),
    "heads across tiles": dict(rows=100, keys=100, heads=2, hd=128, tile=64, cap=8.0, slopes=1),
    "transposed": dict(rows=140, keys=140, heads=2, hd=64, v_trans=1, cap=8.0, spans=_documents(140, [50])),
    "odd tiles": dict(rows=130, keys=171, heads=3, hd=64, row_tile=50, q_pos0=41, cap=8.0, slopes=1, spans=_window(130, 90, first=41)),
    "tiles of sixteen": dict(rows=60, keys=75, heads=2, hd=128, row_tile=16, causal=0, cap=8.0, spans=_holes(60, 75, 4)),
    "capped at a thousand": dict(rows=130, keys=130, heads=2, hd=128, cap=1000.0, std=4.0),
    "capped at half a million": dict(rows=130, keys=130, heads=2, hd=64, cap=5e5, std=4.0),
    "capped at a million, slopes": dict(rows=70, keys=70, heads=2, hd=128, cap=1e6, slopes=1),
    "more blocks than compute units": dict(rows=1100, keys=1100, heads=8, hd=64, spans=_documents(1100, [300, 310, 900])),
    "more of odd heads": dict(rows=1000, keys=300, heads=9, hd=64, causal=0, slopes=1, k_pos0=100),
    "blocks without an order": dict(rows=8300, keys=40, heads=1, hd=64, causal=0, cap=6.0, spans=_holes(8300, 40, 3)),
}


class Case:
    def __init__(self, c, dtype, seed=0):
        self.c = c = {**dict(tile=0, row_tile=0, causal=1, cap=0.0, slopes=0, spans=None, q_pos0=0, k_pos0=0, v_trans=0, std=2.0), **c}
        rng = np.random.default_rng(seed)
        d = c["heads"] * c["hd"]
        self.dtype, self.d = dtype, d
        self.q = rounded(rng.standard_normal((c["rows"], d)) * c["std"], dtype)
        self.k, self.v = (rounded(rng.standard_normal((c["keys"], d)), dtype) for _ in range(2))
        self.do = rounded(rng.standard_normal((c["rows"], d)), dtype)
        self.slopes = 2.0 ** -(1.0 + np.arange(c["heads"])) if c["slopes"] else None
        self.spans = None if c["spans"] is None else np.asarray(c["spans"]).astype(np.int64)
        self.scale = float(np.float32(1 / math.sqrt(c["hd"])))
        self.cap = float(np.float32(c["cap"]))
        self.ok = H.visible(c["rows"], c["keys"], c["q_pos0"], c["k_pos0"], c["causal"], self.spans)

    def rule(self):
        c = self.c
        return dict(head_dim=c["hd"], scale=self.scale, causal=c["causal"], score_cap=c["cap"], slopes=c["slopes"], spans=int(self.spans is not None),
                    q_pos0=c["q_pos0"], v_trans=c["v_trans"])

    def add(self, g):
        """Input vertices (Q, K, V, dO tiles, slopes, spans) and the tiles' shape."""
        c = self.c
        rt, ct = c["row_tile"] or c["tile"] or max(c["rows"], c["keys"]), c["tile"] or self.d
        self.rt, self.ct = rt, ct
        self.nq, self.nkv, self.nc = -(-c["rows"] // rt), -(-c["keys"] // rt), -(-self.d // ct)
        self.Q, self.K, self.dO = (g.grid(a, rt, ct) for a in (self.q, self.k, self.do))
        self.V = g.grid(self.v, rt, ct, transposed=bool(c["v_trans"]))
        self.extra = [g.inp(self.slopes, "f32")] if c["slopes"] else []
        if self.spans is not None:
            self.extra += g.grid(self.spans, rt, 2, "i32")
        return g

    def block(self, g, finish, keys=None):
        c = self.c
        a, b = keys or (0, self.nkv)
        cols, code = (self.d, None) if finish else (self.d + 2 * c["heads"], "f32")
        return g.op(B.TN_OP_ATTN_BLOCK, self.Q + self.K[a * self.nc:b * self.nc] + self.V[a * self.nc:b * self.nc] + self.extra, c["rows"], cols, code,
                    n_q_tiles=self.nq, n_kv_tiles=b - a, n_col_tiles=self.nc, k_pos0=c["k_pos0"] + a * self.rt, finish=finish, **self.rule())

    def join(self, g, parts, finish, dtype=None):
        c = self.c
        return g.op(B.TN_OP_ATTN_COMBINE, parts, c["rows"], c["heads"] if finish == 2 else self.d, "f32" if finish == 2 else dtype, head_dim=c["hd"],
                    hpg=c["heads"], finish=finish)

    def reverse(self, g, part, parts=None):
        """(O tiles' vertex list, log-sum-exps, dQ, dK, dV) behind a partial; statistics from O, or from `parts`, partials of all rows."""
        c = self.c
        par = dict(head_dim=c["hd"], hpg=c["heads"])
        cut = lambda n, s: [(x, min(x + s, n)) for x in range(0, n, s)]  # noqa: E731
        o = [g.op(B.TN_OP_ATTN_COMBINE, [part], r1 - r0, c1 - c0, row0=r0, col0=c0, finish=1, **par)
             for r0, r1 in cut(c["rows"], self.rt) for c0, c1 in cut(self.d, self.ct)]
        lse = [g.op(B.TN_OP_ATTN_COMBINE, [part], r1 - r0, c["heads"], "f32", row0=r0, finish=2, **par) for r0, r1 in cut(c["rows"], self.rt)]
        stats = [g.op(B.TN_OP_ATTN_BWD, o[i * self.nc:(i + 1) * self.nc] + self.dO[i * self.nc:(i + 1) * self.nc] + [lse[i]], r1 - r0, 2 * c["heads"], "f32",
                      mode=4, n_q_tiles=1, n_col_tiles=self.nc, head_dim=c["hd"]) for i, (r0, r1) in enumerate(cut(c["rows"], self.rt))]
        if parts:
            stats = [g.op(B.TN_OP_ATTN_BWD, parts + self.dO[i * self.nc:(i + 1) * self.nc], r1 - r0, 2 * c["heads"], "f32", mode=4, nk=len(parts), row0=r0,
                          n_q_tiles=1, n_col_tiles=self.nc, head_dim=c["hd"]) for i, (r0, r1) in enumerate(cut(c["rows"], self.rt))]
        grads = [g.op(B.TN_OP_ATTN_BWD, self.Q + self.K + self.V + self.dO + stats + self.extra, c["rows"] if mode == 1 else c["keys"], self.d, mode=mode,
                      n_q_tiles=self.nq, n_kv_tiles=self.nkv, n_col_tiles=self.nc, k_pos0=c["k_pos0"], **self.rule()) for mode in (1, 2, 3)]
        return o, lse, grads

    def exact(self, grad=False):
        c = self.c
        q, k, v = (torch.tensor(a, requires_grad=grad) for a in (self.q, self.k, self.v))
        o, lse = H.attention(q, k, v, c["hd"], self.scale, self.ok, self.cap, self.slopes, c["q_pos0"], c["k_pos0"])
        if not grad:
            return o.numpy(), lse.numpy()
        return (o.detach().numpy(), lse.numpy()) + tuple(x.numpy() for x in torch.autograd.grad(o, (q, k, v), torch.tensor(self.do)))

    def bounds(self, grad=False, rounded_o=True, weights=-16):
        """weights: what of a weight (2 to this) rounding to bf16 loses: once in finished rows, else what two of them leave."""
        c, b = self.c, self.dtype == "bf16"
        t = torch.tensor
        x = H.attention_bounds(t(self.q), t(self.k), t(self.v), c["hd"], self.scale, self.ok, 2.0 ** (-8 if b else -24), 2.0 ** weights if b else 0.0, self.cap,
                               self.slopes, c["q_pos0"], c["k_pos0"], t(self.do) if grad else None, rounded_o, cap_sized=b and self.cap <= 1024.0)
        return {n: a.numpy() for n, a in x.items()}


def _within(got, ref, tol, what):
    fine = np.isfinite(ref)
    assert (got[~fine] == ref[~fine]).all(), what
    off = np.abs(got[fine] - ref[fine])
    over, worst = off - tol[fine], np.max(off / np.maximum(tol[fine], 1e-30)) if fine.any() else 0.0
    assert (over <= 0).all(), f"{what}: {worst:.2f} times its bound"
    return worst


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", CASES)
def test_forward(name, dtype):
    x = Case(CASES[name], dtype)
    g = x.add(Graph(dtype))
    part = x.block(g, 0)
    parts = [x.block(g, 0, (i, i + 1)) for i in range(x.nkv)]  # a vertex per row tile of keys, joined
    whole, joined, lse, split, lse2 = g.run([x.block(g, 1), x.join(g, [part], 1), x.join(g, [part], 2), x.join(g, parts, 1), x.join(g, parts, 2)])
    o, l = x.exact()
    tol = x.bounds()
    for a, n in ((whole, "whole"), (joined, "joined"), (split, "split")):
        _within(a, o, (x.bounds(weights=-8) if n == "whole" else tol)["o"], n)
        assert (a[~x.ok.numpy().any(1)] == 0).all()
    _within(lse, l, tol["lse"], "lse")
    _within(lse2, l, tol["lse"], "lse of the split")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("stats", ["O", "a partial", "partials"])
@pytest.mark.parametrize("name", CASES)
def test_reverse(name, stats, dtype):
    x = Case(CASES[name], dtype, 1)
    g = x.add(Graph(dtype))
    part = x.block(g, 0)
    parts = {"O": None, "a partial": [part]}.get(stats) if stats != "partials" else [x.block(g, 0, (i, i + 1)) for i in range(x.nkv)]
    _, _, grads = x.reverse(g, part, parts)
    got = g.run(grads)
    ref, tol = x.exact(True)[2:], x.bounds(True, stats == "O")
    for n, a, r in zip(("dq", "dk", "dv"), got, ref):
        _within(a, r, tol[n], n)
    sees = x.ok.numpy()
    assert (got[0][~sees.any(1)] == 0).all() and (got[1][~sees.any(0)] == 0).all() and (got[2][~sees.any(0)] == 0).all()


def test_gradients_against_differences():
    x = Case(CASES["documents in tiles"], "f32", 2)
    x.cap = 4.0
    x.c["cap"] = 4.0
    g = x.add(Graph())
    got = g.run(x.reverse(g, x.block(g, 0))[2])
    rng, h = np.random.default_rng(3), 1e-4

    def loss():
        return float((x.exact()[0] * x.do).sum())

    for name, grad in zip("qkv", got):
        for _ in range(3):
            step, a = rng.standard_normal(grad.shape), getattr(x, name)
            setattr(x, name, a + h * step)
            up = loss()
            setattr(x, name, a - h * step)
            slope = (up - loss()) / (2 * h)
            setattr(x, name, a)
            assert abs(slope - (grad * step).sum()) <= 1e-4 * np.abs(grad * step).sum()  # 1e-5 of fp32 gradients, h^2 of the difference


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["documents", "documents in tiles", "window", "prefix", "holes", "behind a cache"])
def test_what_a_row_does_not_see_may_be_anything(name, dtype):
    """Infinities and NaN in keys, values, queries and gradients that a row does not see leave it alone."""
    x = Case(CASES[name], dtype, 4)
    ok = x.ok.numpy()
    g = x.add(Graph(dtype))
    o, lse, grads = x.reverse(g, x.block(g, 0))
    clean = g.run([x.block(g, 1), lse[0]] + grads)
    hurt_k, hurt_q = np.zeros(x.c["keys"], bool), np.zeros(x.c["rows"], bool)
    hurt_k[[10 if name == "behind a cache" else x.c["keys"] // 2 + 3, x.c["keys"] - 1]] = True
    hurt_q[[x.c["rows"] // 3, x.c["rows"] - 1]] = True
    y = Case(CASES[name], dtype, 4)
    y.v[hurt_k] = np.inf
    y.v[np.flatnonzero(hurt_k)[0], 5] = np.nan
    y.k[np.flatnonzero(hurt_k)[-1]] = np.nan
    y.q[np.flatnonzero(hurt_q)[0]] = np.nan
    y.do[np.flatnonzero(hurt_q)[-1]] = -np.inf
    g = y.add(Graph(dtype))
    o, lse, grads = y.reverse(g, y.block(g, 0))
    got = g.run([y.block(g, 1), lse[0]] + grads)
    safe_q = ~(ok[:, hurt_k].any(1) | hurt_q)  # rows whose results cannot depend on what was hurt
    touched = ~safe_q
    safe_k = ~(ok[touched].any(0) | hurt_k)
    assert safe_q.any()
    tolg = dict(x.bounds(True), o=x.bounds(weights=-8)["o"])  # finished rows
    for n, a, c, safe in (("o", got[0], clean[0], safe_q), ("dq", got[2], clean[2], safe_q), ("dk", got[3], clean[3], safe_k), ("dv", got[4], clean[4], safe_k)):
        assert np.isfinite(a[safe]).all(), n
        assert (np.abs(a - c)[safe] <= 2 * tolg[n][safe]).all(), n  # both within the bound of the exact values
    # and what sees them is not silently finite
    assert not np.isfinite(got[0][ok[:, np.flatnonzero(hurt_k)[0]]]).all() or not ok[:, np.flatnonzero(hurt_k)[0]].any()




@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_padding_behind_the_last_sequence(dtype):
    """A padded batch: rows behind the sequences hold NaN and see nothing; they give zeros and change nothing."""
    c = dict(rows=200, keys=200, heads=2, hd=128, spans=_documents(200, [70], 61), cap=20.0)
    x = Case(c, dtype, 5)
    for a in (x.q, x.k, x.v, x.do):
        a[139:] = np.nan
    g = x.add(Graph(dtype))
    o, lse, grads = x.reverse(g, x.block(g, 0))
    got = g.run([x.block(g, 1)] + grads)
    y = Case(dict(rows=139, keys=139, heads=2, hd=128, spans=_documents(139, [70]), cap=20.0), dtype, 5)
    for n in ("q", "k", "v", "do"):
        setattr(y, n, getattr(x, n)[:139])
    ref, tol = y.exact(True), dict(y.bounds(True), o=y.bounds(weights=-8)["o"])  # finished rows
    for n, a, r in (("o", got[0], ref[0]), ("dq", got[1], ref[2]), ("dk", got[2], ref[3]), ("dv", got[3], ref[4])):
        _within(a[:139], r, tol[n], n)
        assert (a[139:] == 0).all(), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,heads,hd,parts,col0,cols", [(1, 4, 64, 16, 0, 256), (1, 4, 64, 15, 0, 256), (1, 2, 128, 300, 0, 256), (3, 6, 64, 33, 128, 192), (5, 2, 128, 19, 128, 128),
                                                            (2, 2, 1024, 17, 0, 2048), (3, 4, 20, 70, 20, 40), (1, 3, 64, 20, 0, 192), (2, 2, 64, 12, 32, 64)])
def test_joins_of_few_rows(rows, heads, hd, parts, col0, cols, dtype):
    """Partials as any attention leaves them, some of a row that saw nothing, one row that no partial has seen a key of."""
    rng = np.random.default_rng(9)
    d = heads * hd
    P = rng.standard_normal((parts, rows, d + 2 * heads)).astype(np.float32)
    P[..., d:d + heads] *= 20
    P[..., d + heads:] = np.abs(P[..., d + heads:]) + 1
    empty = rng.random((parts, rows)) < 0.3
    empty[:, -1] |= rows > 1
    P[empty] = 0
    P[empty, d:d + heads] = -np.inf
    g = Graph(dtype)
    ins = [g.inp(p, "f32") for p in P]
    out, lse = g.run([g.op(B.TN_OP_ATTN_COMBINE, ins, rows, cols, col0=col0, head_dim=hd, hpg=heads, finish=1),
                      g.op(B.TN_OP_ATTN_COMBINE, ins, rows, heads, "f32", head_dim=hd, hpg=heads, finish=2)])
    P = P.astype(np.float64)
    m, l = P[..., d:d + heads], P[..., d + heads:]
    top = np.where(np.isinf(m.max(0)), 0, m.max(0))
    w = np.exp(m - top)
    den = (w * l).sum(0)
    num = (P[..., :d].reshape(parts, rows, heads, hd) * w[..., None]).sum(0)
    size = (np.abs(P[..., :d]).reshape(parts, rows, heads, hd) * w[..., None]).sum(0)
    safe = np.where(den == 0, 1, den)[..., None]
    ref, size = (a.reshape(rows, d)[:, col0:col0 + cols] for a in (num / safe, size / safe))
    # weights: exponents of up to 80 in 24 bits, 80 units; sums over the partials, a unit each; one rounding to storage
    tol = (parts + 200) * 2.0 ** -24 * size + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref)
    assert (np.abs(out - ref) <= tol).all()
    with np.errstate(divide="ignore"):
        want = top + np.log(den)
    _within(lse, want, (parts + 200) * 2.0 ** -24 * (1 + np.abs(np.where(np.isinf(want), 0, want))), "lse")


@pytest.mark.parametrize("rows,keys,causal", [(2, 2, 1), (3, 3, 1), (40, 2, 0), (64, 3, 0)])
def test_gradients_of_rows_that_see_few_keys(rows, keys, causal):
    """bf16, statistics from partials: the gradients as a whole are off by no more than the two roundings they cannot do without (of dS, and of the
    result: each 2^-8 at most of every value, so 2 * 2^-8 of the 2-norm), which O rounded to bf16 in between would exceed."""
    x = Case(dict(rows=rows, keys=keys, heads=8, hd=64, causal=causal), "bf16", 8)
    x.c["cap"] = 0.0
    x.c["slopes"], x.slopes = 1, np.zeros(8)  # a rule that changes nothing
    g = x.add(Graph("bf16"))
    part = x.block(g, 0)
    got, ref = g.run(x.reverse(g, part, [part])[2]), x.exact(True)[2:]
    for n, a, r in zip(("dq", "dk", "dv"), got, ref):
        assert np.linalg.norm(a - r) <= 2 * 2.0 ** -8 * np.linalg.norm(r), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_order_and_the_static_tables_give_the_same_bits(dtype):
    def once(seed, static=False):
        x = Case(CASES["documents in tiles"], dtype, 6)
        g = x.add(Graph(dtype))
        parts = [x.block(g, 0, (i, i + 1)) for i in range(x.nkv)]
        _, _, grads = x.reverse(g, x.block(g, 0))
        return g.run([x.block(g, 1), x.join(g, parts, 1)] + grads, seed=seed, static=static)

    first = once(1)
    for again in (once(2), once(3), once(4, True)):
        assert all((a == b).all() for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_cache_of_more_than_4_gib(dtype):
    """Heads rotated in a tensor of 4.1 GiB and attended to at its beginning and behind 4 GiB; one vertex is values and source of keys."""
    d, hd, n = 4096, 128, 40
    keys = ((1 << 32) + (1 << 27)) // (d * (4 if dtype == "f32" else 2))
    rng = np.random.default_rng(9)
    g = Graph(dtype)
    cache = torch.zeros((keys, d), dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    first, last = rounded(rng.standard_normal((n, d)), dtype), rounded(rng.standard_normal((n, d)), dtype)
    cache[:n], cache[-n:] = torch.from_numpy(first), torch.from_numpy(last)
    kv = B.tn_taskgraph_add_input(g.tg, B.TN_F32 if dtype == "f32" else B.TN_BF16, keys, d, B.TN_HOST)
    g.host[kv] = cache if dtype == "f32" else cache.view(torch.int16)
    q, do = rounded(rng.standard_normal((2, d)), dtype), rounded(rng.standard_normal((2, d)), dtype)
    spans = np.array([[3, n], [keys - n, keys]])
    scale = float(np.float32(hd ** -0.5))
    Q, dO, S = g.inp(q), g.inp(do), g.inp(spans, "i32")
    K = g.op(B.TN_OP_HEAD_ROPE, [kv], keys, d, head_dim=hd, rope_base=1e4, rope_half=1)
    rule = dict(n_q_tiles=1, n_kv_tiles=1, n_col_tiles=1, head_dim=hd, scale=scale, spans=1, score_cap=20.0)
    out = g.op(B.TN_OP_ATTN_BLOCK, [Q, K, kv, S], 2, d, finish=1, **rule)
    part = g.op(B.TN_OP_ATTN_BLOCK, [Q, K, kv, S], 2, d + 64, "f32", **rule)
    stats = g.op(B.TN_OP_ATTN_BWD, [part, dO], 2, 64, "f32", mode=4, nk=1, n_q_tiles=1, n_col_tiles=1, head_dim=hd)
    dq = g.op(B.TN_OP_ATTN_BWD, [Q, K, kv, dO, stats, S], 2, d, mode=1, **rule)
    got, grad = g.run([out, dq], cap=3 * (1 << 32) + (1 << 28) + (1 << 27))
    freq = H.frequencies(hd, 1e4, 0.0, 0, 1.0, 4.0)
    for row, (rows, lo) in enumerate(((first[3:], 3), (last, keys - n))):
        k = H.head_rotate(torch.tensor(rows), hd, torch.arange(lo, lo + len(rows)), freq, True)
        k = torch.tensor(rounded(k.numpy(), dtype))
        x = torch.tensor(q[row:row + 1], requires_grad=True)
        o, _ = H.attention(x, k, torch.tensor(rows), hd, scale, torch.ones(1, len(rows), dtype=torch.bool), 20.0, None, 0, 0)
        (gq,) = torch.autograd.grad(o, x, torch.tensor(do[row:row + 1]))
        # a wrong row anywhere is an error of the order of 1; the rotated keys' rounding may differ by a step where the sine does
        for a, b in ((got[row], o.detach().numpy()[0]), (grad[row], gq.numpy()[0])):
            assert np.linalg.norm(a - b) <= (1e-5 if dtype == "f32" else 2e-2) * np.linalg.norm(b)
