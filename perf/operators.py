"""What is measured of the operators between the projections of an attention layer: the norm and rotation of each
head of the queries and keys, attention whose scores follow a rule (a cap, a bias by distance, visible spans of
keys), and the gradients of both.

A case is one program of vertices over tensors that lie in GPU memory.  `run` computes it in its plain form, or
(`own`) executes the memgraph that `prepare` compiled, whose inputs lie at their compiled places in the device buffer.
"""
import math

import torch

own = False

DEFAULTS = {
    "dtype": "bf16",
    "heads": 32,
    "head_dim": 128,
    "tile": 0,            # rows and columns of an input tile; 0: the whole tensor is one
    # rotations
    "pos0": 0,
    "norm": True,         # every head normalised, times a gain, before it is rotated
    "half": True,         # pairs (i, i + rotary / 2) instead of (2i, 2i + 1)
    "rotary": 0,          # leading dimensions of a head that are rotated; 0: all
    "base": 10000.0,
    "factor": 0.0,        # > 1: low frequencies divided by it, for contexts longer than `len0`
    "len0": 0,
    "own_positions": 0,   # > 0: rows name their positions: documents of that many rows, each counted from 0
    # attention
    "cap": 0.0,
    "slopes": False,
    "mask": "causal",     # "causal", "documents" (packed, causal inside), "prefix" (seen by everybody, causal behind), "window"
    "mask_size": 0,       # documents: how many; prefix: its length; window: its length
    "padding": 0,         # rows at the end that see nothing
    "split": 0,           # step: keys to a vertex
}
EPS = 1e-6
LOW, HIGH = 1.0, 4.0      # turns within len0 at or below which a frequency is divided by the factor, at or above which it is kept


def listed():
    return [
        # One generated token: the queries of 32 heads, far into a long context.
        dict(name="rotate_token", op="rotate", rows=1, pos0=100000, base=500000.0, factor=8.0, len0=8192),
        # A small fp32 program: interleaved pairs, half of every head rotated.
        dict(name="rotate_toy_f32", op="rotate", dtype="f32", rows=128, heads=4, head_dim=64, tile=64, half=False, rotary=32),
        # The queries of a prompt whose length is no multiple of anything, in the tiles of the prefill programs.
        dict(name="rotate_prompt_1371", op="rotate", rows=1371, tile=512, factor=8.0, len0=512),
        # The queries of the long prefill as packed documents, each with positions of its own.
        dict(name="rotate_documents_16384", op="rotate", rows=16384, own_positions=2048, base=500000.0),
        # Gradients of queries and gain: two short fp32 sequences, and four packed sequences of the fine-tuning step.
        dict(name="rotate_grad_f32", op="rotate_grad", dtype="f32", rows=320, heads=3, head_dim=64, half=False, own_positions=160),
        dict(name="rotate_grad_4x4096", op="rotate_grad", rows=16384, own_positions=4096),
        # A toy fp32 model with a bias by distance.
        dict(name="scores_f32_1024", op="scores", dtype="f32", rows=1024, heads=16, head_dim=64, slopes=True),
        # A prompt whose first 300 tokens all see each other, capped scores.
        dict(name="scores_prompt_1371", op="scores", rows=1371, tile=512, cap=50.0, mask="prefix", mask_size=300),
        # Prefill of 16384 tokens packed from seven documents, the last rows padding.
        dict(name="scores_documents_16384", op="scores", rows=16384, mask="documents", mask_size=7, padding=100),
        # One generated token against a long cache, capped, in blocks of 512 keys that are joined.
        dict(name="scores_token_16384", op="step", keys=16384, cap=50.0, split=512),
        # Forward and reverse pass: two short fp32 sequences packed, and a layer's sequence of 4096 tokens with capped scores.
        dict(name="scores_train_f32", op="scores_train", dtype="f32", rows=320, heads=3, head_dim=64, mask="documents", mask_size=2, slopes=True),
        dict(name="scores_train_4096", op="scores_train", rows=4096, cap=50.0, mask="documents", mask_size=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Rotations and gradients of 1 to 16384 rows, attention of short and long sequences and of single tokens, both
    storage types, odd lengths, every rule."""
    op = rng.choice(["rotate", "rotate", "rotate_grad", "scores", "scores", "scores_train", "scores_train", "step"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    small = dtype == "f32"
    case = dict(op=op, dtype=dtype, heads=rng.choice([1, 3, 4, 8, 9, 16] + ([] if small else [24, 32, 32])))
    if op in ("rotate", "rotate_grad"):
        case.update(head_dim=rng.choice([64, 80, 96, 128, 128, 256]), rows=_log_int(rng, 1, 16384), half=rng.random() < 0.6,
                    norm=op == "rotate_grad" or rng.random() < 0.7, base=rng.choice([10000.0, 500000.0]))
        if case["heads"] * case["head_dim"] > 4096:
            case["heads"] = 4096 // case["head_dim"]
        if rng.random() < 0.3:
            case["rotary"] = case["head_dim"] // rng.choice([2, 4])
        if rng.random() < 0.4:
            case.update(factor=rng.choice([2.0, 8.0]), len0=rng.choice([512, 8192]))
        if rng.random() < 0.5:
            case["own_positions"] = _log_int(rng, 1, 4096)
        else:
            case["pos0"] = rng.choice([0, rng.randint(1, 200000)])
        return case
    case["head_dim"] = rng.choice([64, 128, 128])
    if rng.random() < 0.5:
        case["cap"] = rng.choice([20.0, 30.0, 50.0])
    if rng.random() < 0.3:
        case["slopes"] = True
    if op == "step":
        keys = _log_int(rng, 1, 16384)
        case.update(keys=keys, split=rng.choice([256, 512, 512, 1024]))
        if rng.random() < 0.4:
            case.update(mask="window", mask_size=_log_int(rng, 1, keys))
        return case
    rows = _log_int(rng, 1, {"scores": 8192, "scores_train": 4096}[op] // (4 if small else 1))
    case["rows"] = rows
    mask = rng.choice(["causal", "documents", "documents", "prefix", "window"])
    if mask == "documents":
        case.update(mask=mask, mask_size=min(rows, rng.randint(1, 12)), padding=rng.choice([0, 0, rows // 16]))
    elif mask != "causal":
        case.update(mask=mask, mask_size=_log_int(rng, 1, rows))
    if rng.random() < 0.4:
        case["tile"] = rng.choice([t for t in (64, 128, 256, 384, 512) if t % case["head_dim"] == 0 and case["heads"] * case["head_dim"] % t == 0] or [0])
    return case


def _full(case):
    return {**DEFAULTS, **case}


# ---- the data ------------------------------------------------------------------------------------

def _bounds(c):
    """Rows at which the packed documents begin, and the end of the last: lengths that differ up to threefold."""
    n, rows = c["mask_size"], c["rows"] - c["padding"]
    weights = [1.0 + 2.0 * ((i * 0.6180339887498949) % 1.0) for i in range(n)]
    ends, total = [], 0.0
    for w in weights:
        total += w
        ends.append(int(round(rows * total / sum(weights))))
    return [0] + ends


def _spans(c):
    """Per query row the first visible key and the one behind the last, or None where the causal rule says it all."""
    if c["op"] == "step":
        if c["mask"] != "window":
            return None
        return torch.tensor([[c["keys"] - c["mask_size"], c["keys"]]], dtype=torch.int32)
    rows = c["rows"]
    if c["mask"] == "causal":
        return None
    at = torch.arange(rows)
    if c["mask"] == "documents":
        s = torch.zeros(rows, 2, dtype=torch.int32)
        b = _bounds(c)
        for lo, hi in zip(b, b[1:]):
            s[lo:hi, 0], s[lo:hi, 1] = lo, hi
        return s
    if c["mask"] == "prefix":
        return torch.stack([torch.zeros_like(at), torch.clamp(at + 1, min=c["mask_size"])], 1).int()
    return torch.stack([torch.clamp(at - c["mask_size"] + 1, min=0), torch.full_like(at, rows)], 1).int()


def _is_causal(c):
    return c["op"] != "step" and c["mask"] != "prefix"


def _visible_pairs(c):
    keys = c["keys"] if c["op"] == "step" else c["rows"]
    rows = 1 if c["op"] == "step" else c["rows"]
    s = _spans(c)
    lo = s[:, 0].long() if s is not None else torch.zeros(rows, dtype=torch.long)
    hi = s[:, 1].long() if s is not None else torch.full((rows,), keys)
    if _is_causal(c):
        hi = torch.minimum(hi, torch.arange(rows) + 1)
    return int(torch.clamp(hi - lo, min=0).sum())


def _data(case, seed):
    """Whole tensors on the GPU, in storage type."""
    c = _full(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    d = c["heads"] * c["head_dim"]

    def normal(rows, cols, std=1.0, mean=0.0):
        return (torch.randn(rows, cols, generator=g, device="cuda") * std + mean).to(kind)

    t = {}
    if c["op"] in ("rotate", "rotate_grad"):
        t["x"] = normal(c["rows"], d)
        if c["norm"]:
            t["gain"] = normal(1, c["head_dim"], 0.1, 1.0)
        if c["own_positions"]:
            t["positions"] = (torch.arange(c["rows"], device="cuda", dtype=torch.int32) % c["own_positions"]).reshape(-1, 1)
        if c["op"] == "rotate_grad":
            t["dy"] = normal(c["rows"], d)
        return t
    rows, keys = (1, c["keys"]) if c["op"] == "step" else (c["rows"], c["rows"])
    t["q"], t["k"], t["v"] = normal(rows, d, 2.0), normal(keys, d), normal(keys, d)  # scores with a deviation of 2
    if c["slopes"]:
        t["slopes"] = 2.0 ** (-8.0 * (torch.arange(c["heads"], device="cuda", dtype=torch.float32) + 1) / c["heads"]).reshape(1, -1)
    s = _spans(c)
    if s is not None:
        t["spans"] = s.cuda()
    if c["op"] == "scores_train":
        t["do"] = normal(rows, d)
    return t


def _cut(n, step):
    return [(a, min(a + step, n)) for a in range(0, n, step)] if step else [(0, n)]


# ---- the program of vertices ---------------------------------------------------------------------

class Program:
    """A taskgraph, compiled with room for every tensor, and its executor: the inputs lie at their compiled places in the
    device buffer, and so do the results when it has run."""

    def __init__(self):
        from paper_2405_16283_amd import binding
        self.B = binding
        self.tg = binding.tn_taskgraph_create()
        self.mg = self.ex = None
        self.inputs = {}

    def inp(self, tensor):
        B = self.B
        code = {torch.float32: B.TN_F32, torch.bfloat16: B.TN_BF16, torch.int32: B.TN_I32}[tensor.dtype]
        v = B.tn_taskgraph_add_input(self.tg, code, tensor.shape[0], tensor.shape[1], B.TN_DEVICE)
        self.inputs[v] = tensor
        return v

    def grid(self, tensor, tile, cols=True):
        """Input vertices of the tensor's tiles, by rows of tiles."""
        return [[self.inp(tensor[r0:r1, c0:c1]) for c0, c1 in _cut(tensor.shape[1], tile if cols else 0)] for r0, r1 in _cut(tensor.shape[0], tile)]

    def op(self, kind, ins, code, rows, cols, **params):
        return self.B.tn_taskgraph_add_op(self.tg, kind, self.B.tn_op_params(**params), ins, code, rows, cols)

    def load(self):
        B = self.B
        n = B.tn_taskgraph_num_vertices(self.tg)
        total = 0
        for v in range(n):
            x = B.tn_taskgraph_vertex(self.tg, v)
            total += (x.desc.rows * x.desc.cols * (2 if x.desc.dtype == B.TN_BF16 else 4) + 255) // 256 * 256
        cap = total + (1 << 20)
        self.mg = B.tn_compile(self.tg, None, cap, B.tn_compile_opts(max_lookahead_bytes=B.UINT64_MAX, next_fit=1))
        place = {}
        for v in range(n):
            m = B.tn_memgraph_vertex(self.mg, v)
            place[v] = (m.offset, m.offset + m.bytes)
        taken = sorted(place.values())
        assert B.tn_memgraph_num_vertices(self.mg) == n and all(a[1] <= b[0] for a, b in zip(taken, taken[1:]))
        self.dev = torch.empty(cap, dtype=torch.uint8, device="cuda")
        self.where = place
        for v, t in self.inputs.items():
            self.view(v).copy_(t)
        self.inputs = {}
        self.streams = [torch.cuda.Stream() for _ in range(3)]
        torch.cuda.synchronize()
        s = [x.cuda_stream for x in self.streams]
        self.ex = B.tn_executor_create(self.mg, self.dev.data_ptr(), cap, 0, 0, s[:1], s[1], s[2])
        self.opts = B.tn_exec_opts(policy=B.TN_POLICY_BY_ORDER, max_batch=1920, queue_depth=8)
        self.none = B.ptr_array([0] * n)

    def view(self, v):
        """The tensor of a vertex where it lies."""
        B = self.B
        x = B.tn_taskgraph_vertex(self.tg, v).desc
        lo, hi = self.where[v]
        return self.dev[lo:hi].view({B.TN_F32: torch.float32, B.TN_BF16: torch.bfloat16, B.TN_I32: torch.int32}[x.dtype]).reshape(x.rows, x.cols)

    def execute(self):
        self.B.tn_execute(self.ex, self.none, self.none, self.opts)

    def __del__(self):
        if self.ex is not None:
            torch.cuda.synchronize()
            self.B.tn_executor_destroy(self.ex)
        if self.mg is not None:
            self.B.tn_memgraph_destroy(self.mg)
        self.B.tn_taskgraph_destroy(self.tg)


def _rotation(c):
    return dict(pos0=c["pos0"], head_dim=c["head_dim"], rotary_dim=c["rotary"], rope_half=int(c["half"]), rope_base=c["base"],
                positions=int(c["own_positions"] > 0), norm=int(c["norm"]), eps=EPS, rope_factor=c["factor"], rope_len0=c["len0"],
                rope_low=LOW, rope_high=HIGH)


def _build(c, t):
    p = Program()
    B = p.B
    code = B.TN_F32 if c["dtype"] == "f32" else B.TN_BF16
    hd, heads = c["head_dim"], c["heads"]
    d, flat = heads * hd, lambda grid: [v for row in grid for v in row]
    if c["op"] in ("rotate", "rotate_grad"):
        gain = [p.inp(t["gain"])] if c["norm"] else []
        outs = {"y": []} if c["op"] == "rotate" else {"dx": []}
        pieces = []
        for r0, r1 in _cut(c["rows"], c["tile"]):
            pos = [p.inp(t["positions"][r0:r1])] if c["own_positions"] else []
            for c0, c1 in _cut(d, c["tile"]):
                par = {**_rotation(c), "pos0": c["pos0"] + (0 if pos else r0)}
                x = p.inp(t["x"][r0:r1, c0:c1])
                if c["op"] == "rotate":
                    outs["y"].append(p.op(B.TN_OP_HEAD_ROPE, [x] + gain + pos, code, r1 - r0, c1 - c0, **par))
                    continue
                dy = p.inp(t["dy"][r0:r1, c0:c1])
                outs["dx"].append(p.op(B.TN_OP_HEAD_ROPE_BWD, [dy, x] + gain + pos, code, r1 - r0, c1 - c0, **par))
                pieces.append(p.op(B.TN_OP_HEAD_ROPE_BWD, [dy, x] + gain + pos, B.TN_F32, (r1 - r0 + 31) // 32, hd, mode=1, **par))
        if pieces:
            outs["dgain"] = [p.op(B.TN_OP_COL_SUM, pieces, B.TN_F32, 1, hd)]
        p.load()
        return p, outs
    keys = t["k"].shape[0]
    rule = dict(head_dim=hd, scale=1.0 / math.sqrt(hd), causal=int(_is_causal(c)), score_cap=c["cap"], slopes=int(c["slopes"]), spans=int("spans" in t))
    slopes = [p.inp(t["slopes"])] if c["slopes"] else []
    if c["op"] == "step":
        q = p.inp(t["q"])
        spans = [p.inp(t["spans"])] if "spans" in t else []
        blocks = [p.op(B.TN_OP_ATTN_BLOCK, [q, p.inp(t["k"][a:b]), p.inp(t["v"][a:b])] + slopes + spans, B.TN_F32, 1, d + 2 * heads, n_q_tiles=1,
                       n_kv_tiles=1, n_col_tiles=1, q_pos0=keys - 1, k_pos0=a, **rule) for a, b in _cut(keys, c["split"])]
        outs = {"o": [p.op(B.TN_OP_ATTN_COMBINE, blocks, code, 1, d, head_dim=hd, hpg=heads, finish=1)]}
        p.load()
        return p, outs
    rows = c["rows"]
    q, k, v = (p.grid(t[n], c["tile"]) for n in "qkv")
    spans = flat(p.grid(t["spans"], c["tile"], cols=False)) if "spans" in t else []
    par = dict(n_q_tiles=len(q), n_kv_tiles=len(k), n_col_tiles=len(q[0]), **rule)
    if c["op"] == "scores":
        outs = {"o": [p.op(B.TN_OP_ATTN_BLOCK, flat(q) + flat(k) + flat(v) + slopes + spans, code, rows, d, finish=1, **par)]}
        p.load()
        return p, outs
    do = p.grid(t["do"], c["tile"])
    part = p.op(B.TN_OP_ATTN_BLOCK, flat(q) + flat(k) + flat(v) + slopes + spans, B.TN_F32, rows, d + 2 * heads, **par)
    r_, c_ = _cut(rows, c["tile"]), _cut(d, c["tile"])
    o = [[p.op(B.TN_OP_ATTN_COMBINE, [part], code, r1 - r0, c1 - c0, row0=r0, col0=c0, head_dim=hd, hpg=heads, finish=1) for c0, c1 in c_] for r0, r1 in r_]
    stats = [p.op(B.TN_OP_ATTN_BWD, [part] + do[i], B.TN_F32, r1 - r0, 2 * heads, mode=4, nk=1, row0=r0, n_q_tiles=1, n_col_tiles=len(c_), head_dim=hd)
             for i, (r0, r1) in enumerate(r_)]
    ins = flat(q) + flat(k) + flat(v) + flat(do) + stats + slopes + spans
    outs = {"o": flat(o)}
    for mode, name in ((1, "dq"), (2, "dk"), (3, "dv")):
        outs[name] = [p.op(B.TN_OP_ATTN_BWD, ins, code, rows, d, mode=mode, **par)]
    p.load()
    return p, outs


class State:
    pass


def prepare(case, seed):
    s = State()
    s.c = _full(case)
    s.t = _data(case, seed)
    s.program = None
    if own:
        s.program, outs = _build(s.c, s.t)
        s.results = {name: [s.program.view(v) for v in vs] for name, vs in outs.items()}
        s.t = None  # the inputs lie in the program's buffer
    return s


def run(state):
    if state.program is not None:
        state.program.execute()
        return state.results
    return _plain(state.c, state.t)


# ---- the plain form: 32 bits -----------------------------------------------------------------------

def _tiles(c, full):
    """The result in the pieces in which the program of vertices leaves it."""
    return [full[r0:r1, c0:c1] for r0, r1 in _cut(full.shape[0], c["tile"]) for c0, c1 in _cut(full.shape[1], c["tile"])]


def _frequencies(c):
    """Radians per position of every rotated pair, in 64 bits."""
    rd = c["rotary"] or c["head_dim"]
    f = c["base"] ** (-torch.arange(0, rd, 2, dtype=torch.float64, device="cuda") / rd)
    if c["factor"] > 1:
        turns = c["len0"] * f / (2 * math.pi)
        kept = torch.clamp((turns - LOW) / (HIGH - LOW), 0, 1)
        f = f * kept + f / c["factor"] * (1 - kept)
    return f


def _turn(c, t, back=False):
    """(cosine, sine) of every row and rotated pair, [rows, 1, pairs]."""
    rows = t["x"].shape[0]
    at = t["positions"][:, 0].double() if "positions" in t else torch.arange(rows, device="cuda", dtype=torch.float64)
    a = (at + c["pos0"])[:, None] * _frequencies(c)
    return a.cos().float()[:, None], (-a.sin() if back else a.sin()).float()[:, None]


def _rotated(c, x, cos, sin):
    """x: [rows, heads, head_dim]"""
    n = cos.shape[-1]
    if c["half"]:
        a, b = x[..., :n], x[..., n:2 * n]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., 2 * n:]], -1)
    a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., 2 * n:]], -1)


def _plain_rotate(c, t):
    x = t["x"].float().reshape(c["rows"], c["heads"], c["head_dim"])
    if c["norm"]:
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    if c["op"] == "rotate":
        if c["norm"]:
            x = x * r * t["gain"].float()
        return {"y": _tiles(c, _rotated(c, x, *_turn(c, t)).flatten(1).to(t["x"].dtype))}
    u = _rotated(c, t["dy"].float().reshape(x.shape), *_turn(c, t, back=True))
    n = x * r
    du = u * t["gain"].float()
    dx = r * (du - n * (du * n).mean(-1, keepdim=True))
    return {"dx": _tiles(c, dx.flatten(1).to(t["x"].dtype)), "dgain": [(u * n).sum((0, 1)).reshape(1, -1)]}


def _plain_scores(c, t):
    rows, keys, hd = t["q"].shape[0], t["k"].shape[0], c["head_dim"]
    kind, scale = t["q"].dtype, 1.0 / math.sqrt(hd)
    qp = torch.arange(keys - rows, keys, device="cuda")[:, None]
    kp = torch.arange(keys, device="cuda")[None]
    seen = None
    if _is_causal(c):
        seen = kp <= qp
    if "spans" in t:
        inside = (kp >= t["spans"][:, :1]) & (kp < t["spans"][:, 1:])
        seen = inside if seen is None else seen & inside
    train = c["op"] == "scores_train"
    outs = {n: [] for n in (("o", "dq", "dk", "dv") if train else ("o",))}
    by_head = lambda x, h: x.reshape(x.shape[0], -1, hd)[:, h].float().transpose(0, 1)  # noqa: E731
    some = max(1, (1 << 28) // (rows * keys))  # heads at a time: scores of 1 GiB
    for h0 in range(0, c["heads"], some):
        at = slice(h0, h0 + some)
        q, k, v = (by_head(t[n], at).contiguous() for n in "qkv")
        s = torch.bmm(q, k.transpose(1, 2).contiguous()) * scale
        if c["cap"]:
            tanh = torch.tanh(s / c["cap"])
            s = c["cap"] * tanh
        if c["slopes"]:
            s = s - t["slopes"][0, at, None, None] * (qp - kp).abs()
        if seen is not None:
            s = s.masked_fill(~seen, -math.inf)
        m = s.amax(-1, keepdim=True)
        p = torch.exp(s - m.masked_fill(m == -math.inf, 0.0))
        total = p.sum(-1, keepdim=True)
        p = p / total.masked_fill(total == 0, 1.0)
        o = torch.bmm(p, v)
        outs["o"].append(o.to(kind))
        if train:
            do = by_head(t["do"], at).contiguous()
            ds = p * (torch.bmm(do, v.transpose(1, 2).contiguous()) - (do * o).sum(-1, keepdim=True))
            if c["cap"]:
                ds = ds * (1 - tanh * tanh)
            outs["dq"].append((torch.bmm(ds, k) * scale).to(kind))
            outs["dk"].append((torch.bmm(ds.transpose(1, 2).contiguous(), q) * scale).to(kind))
            outs["dv"].append(torch.bmm(p.transpose(1, 2).contiguous(), do).to(kind))
    whole = {n: torch.cat(x).transpose(0, 1).reshape(rows, -1) for n, x in outs.items()}
    return {n: _tiles(c, x) if n == "o" and train else [x] for n, x in whole.items()}


def _plain(c, t):
    return _plain_rotate(c, t) if c["op"] in ("rotate", "rotate_grad") else _plain_scores(c, t)


# ---- the definition in 64 bits ---------------------------------------------------------------------

def exact(case, seed):
    c, t = _full(case), _data(case, seed)
    hd, heads = c["head_dim"], c["heads"]
    if c["op"] in ("rotate", "rotate_grad"):
        rd = c["rotary"] or hd
        rows = c["rows"]
        theta = []
        for i in range(rd // 2):
            f = c["base"] ** (-2.0 * i / rd)
            if c["factor"] > 1:
                turns = c["len0"] / (2.0 * math.pi / f)
                if turns <= LOW:
                    f = f / c["factor"]
                elif turns < HIGH:
                    share = (turns - LOW) / (HIGH - LOW)
                    f = f * (share + (1.0 - share) / c["factor"])
            theta.append(f)
        theta = torch.tensor(theta, dtype=torch.float64, device="cuda")
        pos = torch.arange(rows, device="cuda", dtype=torch.float64)
        if c["own_positions"]:
            pos = pos % c["own_positions"]
        unit = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), (pos + c["pos0"])[:, None] * theta)[:, None]
        x = t["x"].double().reshape(rows, heads, hd).requires_grad_(c["op"] == "rotate_grad")
        gain = t["gain"].double().requires_grad_(c["op"] == "rotate_grad") if c["norm"] else None
        n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain if c["norm"] else x
        part = n[..., :rd]
        z = torch.complex(*part.chunk(2, -1)) if c["half"] else torch.complex(part[..., ::2], part[..., 1::2])
        z = z * unit
        turned = torch.cat([z.real, z.imag], -1) if c["half"] else torch.view_as_real(z).flatten(-2)
        y = torch.cat([turned, n[..., rd:]], -1).flatten(1)
        if c["op"] == "rotate":
            return {"y": _tiles(c, y)}
        dx, dgain = torch.autograd.grad(y, (x, gain), t["dy"].double())
        return {"dx": _tiles(c, dx.flatten(1)), "dgain": [dgain]}
    train = c["op"] == "scores_train"
    rows, keys = t["q"].shape[0], t["k"].shape[0]
    row, key = torch.arange(rows, device="cuda") + (keys - rows), torch.arange(keys, device="cuda")
    lo, hi = torch.zeros_like(row), torch.full_like(row, keys)
    if "spans" in t:
        lo, hi = t["spans"][:, 0].long(), t["spans"][:, 1].long()
    if _is_causal(c):
        hi = torch.minimum(hi, row + 1)
    hidden = torch.logical_or(key < lo[:, None], key >= hi[:, None])
    parts = {n: [] for n in (("o", "dq", "dk", "dv") if train else ("o",))}
    for h in range(heads):
        q, k, v = (t[n].reshape(-1, heads, hd)[:, h].double().requires_grad_(train) for n in "qkv")
        s = q.mm(k.t()).div(math.sqrt(hd))
        if c["cap"]:
            s = torch.tanh(s / c["cap"]) * c["cap"]
        if c["slopes"]:
            s = s - t["slopes"][0, h].double() * (row[:, None] - key).abs()
        p = torch.softmax(s.masked_fill(hidden, -1e300), -1).masked_fill(hidden, 0.0)  # a row that sees nothing: zeros
        o = p.mm(v)
        parts["o"].append(o.detach())
        if train:
            for n, grad in zip(("dq", "dk", "dv"), torch.autograd.grad(o, (q, k, v), t["do"].reshape(-1, heads, hd)[:, h].double())):
                parts[n].append(grad)
        del s, p, o
    whole = {n: torch.cat(x, 1) for n, x in parts.items()}
    return {n: _tiles(c, x) if n == "o" and train else [x] for n, x in whole.items()}


# ---- what a pass cannot do without -----------------------------------------------------------------

def work(case):
    c = _full(case)
    e = 4 if c["dtype"] == "f32" else 2
    d = c["heads"] * c["head_dim"]
    if c["op"] in ("rotate", "rotate_grad"):
        n = c["rows"] * d
        extra = 4 * c["rows"] if c["own_positions"] else 0
        if c["op"] == "rotate":
            return {"bytes": float(2 * n * e + extra + c["norm"] * c["head_dim"] * e), "flops": n * (3.0 + 4.0 * c["norm"])}
        return {"bytes": float(3 * n * e + extra + c["head_dim"] * (e + 4)), "flops": n * 14.0}
    rows, keys = (1, c["keys"]) if c["op"] == "step" else (c["rows"], c["rows"])
    pairs = _visible_pairs(c)
    read = keys
    if c["op"] == "step" and c["mask"] == "window":
        read = c["mask_size"]
    train = c["op"] == "scores_train"
    spans = 8 * rows if _spans(c) is not None else 0
    # Q, K, V in and O out; with gradients dO in, dQ, dK and dV out
    elems = (2 * rows + 2 * read) * d + (4 * rows * d if train else 0)
    # two products of the scores' size, and five more for the gradients (scores and probabilities' gradients, dQ, dK, dV)
    return {"bytes": float(elems * e + spans), "flops": (14.0 if train else 4.0) * pairs * d}
