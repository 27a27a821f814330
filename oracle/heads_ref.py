"""Heads and scores in 64 bits: the norm and rotation of query and key heads, and attention whose scores follow a rule (a cap, a
bias by distance, visible spans of keys).  Torch on the CPU, differentiable, from the formulas of turnip.h."""
import math

import torch


def frequencies(rotary_dim, base, factor=0.0, len0=0, low=0.0, high=0.0):
    """Radians per position of every pair."""
    out = []
    for i in range(rotary_dim // 2):
        f = base ** (-2.0 * i / rotary_dim)
        if factor > 1:
            turns = len0 * f / (2 * math.pi)
            share = 0.0 if len0 == 0 else min(1.0, max(0.0, (turns - low) / (high - low)))
            f = share * f + (1 - share) * f / factor
        out.append(f)
    return torch.tensor(out, dtype=torch.float64)


def head_norm(x, head_dim, gain, eps):
    h = x.reshape(x.shape[0], -1, head_dim)
    return (h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps) * gain.reshape(-1)).reshape(x.shape)


def head_rotate(x, head_dim, positions, freq, half, inverse=False):
    """x [rows, heads * head_dim], positions [rows]; the leading 2 len(freq) elements of every head turn."""
    h = x.reshape(x.shape[0], -1, head_dim)
    n = len(freq)
    angle = positions.double()[:, None] * freq * (-1 if inverse else 1)
    z = torch.complex(h[..., :n], h[..., n:2 * n]) if half else torch.complex(h[..., 0:2 * n:2], h[..., 1:2 * n:2])
    z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
    turned = torch.cat([z.real, z.imag], -1) if half else torch.stack([z.real, z.imag], -1).flatten(-2)
    return torch.cat([turned, h[..., 2 * n:]], -1).reshape(x.shape)


def visible(rows, keys, q_pos0, k_pos0, causal, spans=None):
    """[rows, keys]: which keys a row sees."""
    q, k = torch.arange(rows)[:, None] + q_pos0, torch.arange(keys)[None] + k_pos0
    ok = (k <= q) if causal else torch.ones(rows, keys, dtype=torch.bool)
    if spans is not None:
        spans = torch.as_tensor(spans, dtype=torch.int64)
        ok = ok & (k >= spans[:, :1]) & (k < spans[:, 1:])
    return ok


def scores(q, k, scale, cap=0.0, slope=None, q_pos0=0, k_pos0=0):
    """The scores of one head by the rule, before anything is hidden."""
    s = q @ k.T * scale
    if cap:
        s = cap * torch.tanh(s / cap)
    if slope is not None:
        s = s - slope * ((torch.arange(q.shape[0]) + q_pos0)[:, None] - (torch.arange(k.shape[0]) + k_pos0)).abs()
    return s


def attention(q, k, v, head_dim, scale, ok, cap=0.0, slopes=None, q_pos0=0, k_pos0=0):
    """(output [rows, heads * head_dim], log-sum-exp [rows, heads]); zeros and -inf where a row sees nothing."""
    outs, lses = [], []
    for h in range(q.shape[1] // head_dim):
        c = slice(h * head_dim, (h + 1) * head_dim)
        s = scores(q[:, c], k[:, c], scale, cap, None if slopes is None else slopes[h], q_pos0, k_pos0)
        s = s.masked_fill(~ok, -math.inf)
        some = ok.any(1, keepdim=True)
        p = torch.softmax(s.masked_fill(~some, 0.0), 1).masked_fill(~ok, 0.0)
        outs.append(p @ v[:, c])
        lses.append(torch.logsumexp(s.detach(), 1))
    return torch.cat(outs, 1), torch.stack(lses, 1)


def attention_bounds(q, k, v, head_dim, scale, ok, storage, products, cap=0.0, slopes=None, q_pos0=0, k_pos0=0, do=None, rounded_o=True, cap_sized=True):
    """How far correct results may lie from the exact ones, element by element: {"o", "lse"} and with `do` {"dq", "dk", "dv"}.

    Counted are the roundings a kernel makes: of stored results (`storage`: half a step relative to the value, 2^-8 or 2^-24), of weights
    and their gradients where they enter a product (`products`: 2^-16 as two bf16, 0 for fp32), and those of fp32 arithmetic: of
    a score, one unit (2^-24) per term of its sum and a few more for scaling, cap, bias and the exponential; of a sum over n rows, n units;
    a capped score's units are of its own size and, cap_sized, of the cap's (it is formed as cap - 2 cap / (1 + exp(2 z / cap))).
    O enters the reverse pass rounded to storage, or (rounded_o False) as it was before.  Below 2^-126, the smallest normal number, a weight, its gradient or a result may be zero."""
    u, tiny = 2.0 ** -24, 2.0 ** -126
    out = {n: [] for n in ("o", "lse", "dq", "dk", "dv")}
    n = k.shape[0]
    for h in range(q.shape[1] // head_dim):
        c = slice(h * head_dim, (h + 1) * head_dim)
        Q, K, V = q[:, c], k[:, c], v[:, c]
        slope = None if slopes is None else slopes[h]
        raw = (Q.abs() @ K.abs().T) * scale
        s = scores(Q, K, scale, cap, slope, q_pos0, k_pos0)
        size = s.abs() + (cap if cap_sized else 0.0)
        if slope is not None:
            size = size + (s - scores(Q, K, scale, cap)).abs()
        e = u * ((head_dim + 8) * raw + 8 * size + 8)            # of a score
        e = e.masked_fill(~ok, 0.0).amax(1, keepdim=True)
        sm = s.masked_fill(~ok, -math.inf)
        some = ok.any(1, keepdim=True)
        p = torch.softmax(sm.masked_fill(~some, 0.0), 1).masked_fill(~ok, 0.0)
        E = 2 * e + u * (n + 16)                                   # of a weight, relative
        A, o = p @ V.abs(), p @ V
        to = (E + products + u * n) * A + storage * (o.abs() + E * A) + tiny * (1 + V.abs().sum(0))
        out["o"].append(to)
        lse = torch.logsumexp(sm, 1)
        out["lse"].append((E[:, 0] + 4 * u * lse.abs()).nan_to_num(0.0, 0.0, 0.0))
        if do is None:
            continue
        dO = do[:, c]
        t = torch.tanh(Q @ K.T * scale / cap) if cap else torch.zeros_like(s)
        dt = 1 - t * t
        dp, D = dO @ V.T, (dO * o).sum(1, keepdim=True)
        e_dp = (head_dim + 8) * u * (dO.abs() @ V.abs().T)
        to_D = to if rounded_o else (E + products + u * n) * A + tiny * (1 + V.abs().sum(0))
        e_D = (to_D * dO.abs()).sum(1, keepdim=True) + (head_dim + 8) * u * (o.abs() * dO.abs()).sum(1, keepdim=True)
        ds = p * (dp - D) * dt * scale
        e_p = (E + 8 * u) * p + tiny
        e_ds = ds.abs() * (E + products + 16 * u) + p * scale * (dt * (e_dp + e_D) + (dp - D).abs() * (2 * t.abs() * (8 * u + raw * (head_dim + 8) * u / (cap or 1.0)) + 8 * u)) \
            + tiny * (1 + scale * (dp.abs() + D.abs()))
        rows = q.shape[0]
        for name, err, mag, val in (("dq", e_ds @ K.abs(), u * n * (ds.abs() @ K.abs()), ds @ K),
                                    ("dk", e_ds.T @ Q.abs(), u * rows * (ds.abs().T @ Q.abs()), ds.T @ Q),
                                    ("dv", (e_p + products * p).T @ dO.abs(), u * rows * (p.T @ dO.abs()), p.T @ dO)):
            out[name].append(err + mag + storage * (val.abs() + err + mag) + tiny)
    return {k_: torch.stack(x, 1) if k_ == "lse" else torch.cat(x, 1) for k_, x in out.items() if x}


def decoder(cfg, w, heads, probe=None, storage=None):
    """The decoder of lora_ref (float64 arrays by name in `w`: weights, x, adapters where there are any) with the tiler's options on heads
    and scores: `heads` as the harness takes it, its inputs in `w` too (gq.l, gk.l, positions, spans, slopes).  Returns y, and with `probe`
    the gradients of sum(y * probe) by the adapters and x.  storage "bf16": every tensor that the layer stores, and the gradient arriving at
    it, rounded to bf16 (lora_ref's model of a bf16 pipeline): how far from the exact result a correct one may stand."""
    from oracle.lora_ref import _Stored
    S = _Stored.apply if storage == "bf16" else (lambda z: z)
    t = {k: torch.tensor(a, dtype=torch.float64) for k, a in w.items()}
    wanted = [k for k in t if k.split(".")[0] in ("aq", "bq", "av", "bv")] + ["x"]
    for k in wanted:
        t[k].requires_grad_(probe is not None)
    hd, seq = cfg.head_dim, cfg.total_seq
    turned = any(heads.get(k) for k in ("qk_norm", "rope_half", "rotary_dim", "row_positions")) or heads.get("rope_factor", 0) > 1
    freq = frequencies(heads.get("rotary_dim", 0) or hd, float(cfg.rope_base), heads.get("rope_factor", 0.0) if turned else 0.0,
                       heads.get("rope_len0", 0), heads.get("rope_low", 0.0), heads.get("rope_high", 0.0))
    scale = 1 / math.sqrt(hd)

    def norm(x, g):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + cfg.eps) * g

    outs = []
    for b in range(cfg.batch):
        rows = slice(b * seq, (b + 1) * seq)
        x = t["x"][rows]
        pos = t["positions"][rows, 0].detach() if heads.get("row_positions") else torch.arange(seq)
        spans = w["spans"][rows].astype(int) if heads.get("score_spans") else None
        ok = visible(seq, seq, 0, 0, heads.get("score_spans", 0) != 2, spans)
        slopes = t["slopes"].reshape(-1) if heads.get("score_slopes") else None
        for l in range(cfg.layers):
            a = S(norm(x, t[f"g1.{l}"]))
            q, k, v = S(a @ t[f"wq.{l}"]), S(a @ t[f"wk.{l}"]), S(a @ t[f"wv.{l}"])
            if f"aq.{l}" in t:
                q = S(q + S(S(a @ t[f"aq.{l}"]) @ t[f"bq.{l}"]))
                v = S(v + S(S(a @ t[f"av.{l}"]) @ t[f"bv.{l}"]))
            if heads.get("qk_norm"):
                q, k = head_norm(q, hd, t[f"gq.{l}"], cfg.eps), head_norm(k, hd, t[f"gk.{l}"], cfg.eps)
            q, k = (S(head_rotate(z, hd, pos, freq, bool(heads.get("rope_half")))) for z in (q, k))
            o, _ = attention(q, k, v, hd, scale, ok, heads.get("score_cap", 0.0), slopes)
            h1 = S(x + S(S(o) @ t[f"wo.{l}"]))
            bn = S(norm(h1, t[f"g2.{l}"]))
            gate, up = S(bn @ t[f"w1.{l}"]), S(bn @ t[f"w3.{l}"])
            x = S(h1 + S(S(gate * torch.sigmoid(gate) * up) @ t[f"w2.{l}"]))
        outs.append(x)
    y = torch.cat(outs)
    if probe is None:
        return y.detach().numpy()
    grads = torch.autograd.grad((y * torch.tensor(probe)).sum(), [t[k] for k in wanted])
    return y.detach().numpy(), {k: g.numpy() for k, g in zip(wanted, grads)}
