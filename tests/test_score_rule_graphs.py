"""What the operators on heads and scores refuse, and what they are compiled to, on the CPU."""
import pytest

from paper_2405_16283_amd import binding as B


class Tg:
    def __init__(self):
        self.tg = B.tn_taskgraph_create()

    def inp(self, rows, cols, code=B.TN_F32):
        return B.tn_taskgraph_add_input(self.tg, code, rows, cols, B.TN_DEVICE)

    def op(self, kind, ins, rows, cols, code=B.TN_F32, **p):
        return B.tn_taskgraph_add_op(self.tg, kind, B.tn_op_params(**p), ins, code, rows, cols)


@pytest.fixture
def g():
    t = Tg()
    yield t
    B.tn_taskgraph_destroy(t.tg)


def _refused(g, *a, **p):
    n = B.tn_taskgraph_num_vertices(g.tg)
    with pytest.raises(B.TurnipError) as e:
        g.op(*a, **p)
    assert e.value.status == B.TN_ERR_SHAPE and e.value.message
    assert B.tn_taskgraph_num_vertices(g.tg) == n


def test_rotations(g):
    x, gain, pos = g.inp(10, 128), g.inp(1, 64), g.inp(10, 1, B.TN_I32)
    good = dict(head_dim=64, rope_base=1e4, eps=1e-6)
    K, R = B.TN_OP_HEAD_ROPE, B.TN_OP_HEAD_ROPE_BWD
    assert g.op(K, [x], 10, 128, **good) >= 0
    assert g.op(K, [x], 10, 128, mode=1, **good) >= 0
    assert g.op(K, [x, gain, pos], 10, 128, norm=1, positions=1, rotary_dim=32, rope_half=1, rope_factor=4.0, rope_len0=100, rope_low=1.0, rope_high=2.0, **good) >= 0
    assert g.op(R, [x, x, gain, pos], 10, 128, norm=1, positions=1, **good) >= 0
    assert g.op(R, [x, x, gain], 1, 64, norm=1, mode=1, **good) >= 0
    for bad in (dict(head_dim=63), dict(head_dim=0), dict(head_dim=-64), dict(head_dim=256), dict(head_dim=2048), dict(rotary_dim=66), dict(rotary_dim=-2),
                dict(rotary_dim=31), dict(rope_base=0.0), dict(rope_base=float("nan")), dict(rope_base=float("inf")), dict(pos0=-1), dict(mode=2),
                dict(mode=-1), dict(rope_factor=0.5), dict(rope_factor=-2.0), dict(rope_factor=float("inf")), dict(rope_factor=float("nan")),
                dict(rope_factor=2.0, rope_len0=-1), dict(rope_factor=2.0, rope_len0=10), dict(rope_factor=2.0, rope_len0=10, rope_low=2.0, rope_high=1.0),
                dict(rope_factor=2.0, rope_len0=10, rope_low=-1.0, rope_high=1.0), dict(norm=1), dict(positions=1)):
        _refused(g, K, [x], 10, 128, **{**good, **bad})
    _refused(g, K, [x, gain], 10, 128, **good)
    _refused(g, K, [x, gain], 10, 128, norm=1, mode=1, **good)
    _refused(g, K, [x, gain], 10, 128, norm=1, **{**good, "eps": -1.0})
    _refused(g, K, [x, gain], 10, 128, norm=1, **{**good, "eps": float("nan")})
    _refused(g, K, [x, g.inp(1, 128)], 10, 128, norm=1, **good)
    _refused(g, K, [x, g.inp(1, 64, B.TN_BF16)], 10, 128, norm=1, **good)
    _refused(g, K, [x, g.inp(10, 1)], 10, 128, positions=1, **good)          # positions are integers
    _refused(g, K, [x, g.inp(9, 1, B.TN_I32)], 10, 128, positions=1, **good)
    _refused(g, K, [g.inp(10, 128, B.TN_I32)], 10, 128, **good)
    _refused(g, K, [pos, x], 10, 128, positions=1, **good)
    _refused(g, K, [x], 10, 128, B.TN_BF16, **good)
    _refused(g, K, [x], 10, 64, **good)
    _refused(g, K, [x], 10, 128, B.TN_I32, **good)
    _refused(g, R, [x, x], 10, 128, **good)
    _refused(g, R, [x, x, gain], 10, 128, **good)
    _refused(g, R, [g.inp(9, 128), x, gain], 10, 128, norm=1, **good)
    _refused(g, R, [x, x, gain], 1, 128, norm=1, mode=1, **good)
    _refused(g, R, [x, x, gain], 2, 64, norm=1, mode=1, **good)
    _refused(g, B.TN_OP_COL_SUM, [x], 2, 128)
    _refused(g, B.TN_OP_COL_SUM, [x, gain], 1, 128)
    _refused(g, B.TN_OP_COL_SUM, [x], 1, 128, B.TN_BF16)
    assert g.op(B.TN_OP_COL_SUM, [x, g.inp(3, 128)], 1, 128) >= 0


def test_score_rules(g):
    q, k, slopes, spans = g.inp(10, 128), g.inp(20, 128), g.inp(1, 2), g.inp(10, 2, B.TN_I32)
    lse, stats, do = g.inp(10, 2), g.inp(10, 4), g.inp(10, 128)
    A, C, R = B.TN_OP_ATTN_BLOCK, B.TN_OP_ATTN_COMBINE, B.TN_OP_ATTN_BWD
    good = dict(n_q_tiles=1, n_kv_tiles=1, n_col_tiles=1, head_dim=64, scale=0.125)
    assert g.op(A, [q, k, k], 10, 128, finish=1, **good) >= 0
    part = g.op(A, [q, k, k, slopes, spans], 10, 132, score_cap=5.0, slopes=1, spans=1, **good)
    assert g.op(A, [q, k, k, spans], 10, 128, spans=1, finish=1, causal=1, q_pos0=10, **good) >= 0
    for ins, bad in (([q, k, k], dict(score_cap=-1.0)), ([q, k, k], dict(score_cap=float("nan"))), ([q, k, k], dict(score_cap=float("inf"))),
                     ([q, k, k], dict(score_cap=1e-9)), ([q, k, k], dict(finish=2)), ([q, k, k], dict(finish=-1)), ([q, k, k], dict(slopes=1)),
                     ([q, k, k], dict(spans=1)), ([q, k, k, slopes], dict(spans=1)), ([q, k, k, spans], dict(slopes=1)), ([q, k, k, spans, slopes], dict(slopes=1, spans=1)),
                     ([q, k, k, g.inp(10, 2)], dict(spans=1)), ([q, k, k, g.inp(9, 2, B.TN_I32)], dict(spans=1)), ([q, k, k, g.inp(10, 1, B.TN_I32)], dict(spans=1)),
                     ([q, k, k, g.inp(1, 3)], dict(slopes=1)), ([q, k, k, slopes], {}), ([q, k, k], dict(score_cap=5.0, scale=0.0)),
                     ([q, k, k], dict(score_cap=5.0, scale=-1.0)), ([q, k, k], dict(score_cap=5.0, scale=float("nan"))), ([q, k, k], dict(score_cap=5.0, scale=1e-21)), ([q, k, k], dict(score_cap=5.0, scale=1e21)), ([q, k, k], dict(score_cap=5.0, q_pos0=-1)),
                     ([q, k, k], dict(score_cap=5.0, k_pos0=2 ** 30 + 1)), ([q, k, k, spans], dict(spans=1, n_q_tiles=-1)), ([q, k, k, spans], dict(spans=1, n_q_tiles=2 ** 31 - 1)),
                     ([q, g.inp(20, 128, B.TN_I32), k, spans], dict(spans=1))):
        _refused(g, A, ins, 10, 132, **{**good, **bad})
    _refused(g, A, [q, k, k], 10, 132, finish=1, **good)
    _refused(g, A, [q, k, k], 10, 128, B.TN_BF16, finish=1, **good)
    _refused(g, A, [q, k, k], 10, 128, finish=1, **{**good, "scale": 0.0})
    assert g.op(C, [part], 10, 128, head_dim=64, hpg=2, finish=1) >= 0
    assert g.op(C, [part], 4, 2, head_dim=64, hpg=2, finish=2, row0=6) >= 0
    for rows, cols, code, p in ((4, 2, B.TN_F32, dict(row0=7)), (10, 4, B.TN_F32, {}), (10, 2, B.TN_BF16, {}), (10, 2, B.TN_F32, dict(col0=1)), (10, 2, B.TN_F32, dict(row0=-1)),
                                (10, 2, B.TN_F32, dict(finish=3))):
        _refused(g, C, [part], rows, cols, code, **{**dict(head_dim=64, hpg=2, finish=2), **p})
    assert g.op(R, [do, do, lse], 10, 4, mode=4, n_q_tiles=1, n_col_tiles=1, head_dim=64) >= 0
    for ins, rows, cols, p in (([do, do], 10, 4, {}), ([do, do, stats], 10, 4, {}), ([do, k, lse], 10, 4, {}), ([do, do, lse], 10, 2, {}), ([do, do, lse], 9, 4, {}),
                               ([do, do, lse], 10, 4, dict(head_dim=48)), ([do, do, lse], 10, 4, dict(n_q_tiles=2)), ([do, do, lse], 10, 4, dict(mode=5)),
                               ([do, do, spans], 10, 4, dict(spans=1))):
        _refused(g, R, ins, rows, cols, **{**dict(mode=4, n_q_tiles=1, n_col_tiles=1, head_dim=64), **p})
    par = dict(mode=4, nk=2, n_q_tiles=1, n_col_tiles=1, head_dim=64)
    assert g.op(R, [part, part, do], 10, 4, **par) >= 0
    few = g.inp(4, 128)
    assert g.op(R, [part, few], 4, 4, **{**par, "nk": 1, "row0": 6}) >= 0
    for ins, rows, p in (([part, do], 10, {}), ([part, part, do, lse], 10, {}), ([do, do, do], 10, {}), ([part, g.inp(9, 132), do], 10, {}), ([part, part, do], 9, {}),
                         ([part, part, do], 10, dict(row0=1)), ([part, part, do], 10, dict(row0=-1)), ([part, part, do], 10, dict(nk=-2)), ([part, few], 4, dict(nk=1, row0=7))):
        _refused(g, R, ins, rows, 4, **{**par, **p})
    ins = [q, k, k, do, stats, slopes, spans]
    rule = dict(score_cap=5.0, slopes=1, spans=1)
    for mode, rows in ((1, 10), (2, 20), (3, 20)):
        assert g.op(R, ins, rows, 128, mode=mode, **rule, **good) >= 0
        _refused(g, R, ins[:-1], rows, 128, mode=mode, **rule, **good)
        _refused(g, R, ins, rows, 128, mode=mode, trans_a=1, **rule, **good)
    _refused(g, R, [q, k, k, do], 10, 4, mode=0, score_cap=5.0, **good)  # the statistics of a rule come from mode 4
    _refused(g, R, [q, k, k, do, stats], 10, 128, mode=1, score_cap=-5.0, **good)


def test_integers_are_no_operands_of_other_kinds(g):
    i = g.inp(8, 8, B.TN_I32)
    for kind, ins, p in ((B.TN_OP_ADD, [i, i], {}), (B.TN_OP_TRANSPOSE, [i], {}), (B.TN_OP_RMS_STAT, [i], dict(d=8)), (B.TN_OP_GEMM, [i, i], dict(nk=1)),
                         (B.TN_OP_SUM, [i], {}), (B.TN_OP_ROPE, [i], dict(head_dim=4, rope_base=1e4)), (B.TN_OP_SOFTMAX_STAT, [i], dict(scale=1.0)), (B.TN_OP_COL_SUM, [i], {})):
        for code in (B.TN_F32, B.TN_I32):
            for rows, cols in ((8, 8), (8, 1), (8, 2), (1, 8)):
                _refused(g, kind, ins, rows, cols, code, **p)
    with pytest.raises(B.TurnipError):
        B.tn_taskgraph_add_input(g.tg, 3, 8, 8, B.TN_HOST)


def test_integer_inputs_take_four_bytes_each(g):
    x, pos = g.inp(10, 128, B.TN_BF16), g.inp(10, 1, B.TN_I32)
    g.op(B.TN_OP_HEAD_ROPE, [x, pos], 10, 128, B.TN_BF16, head_dim=64, rope_base=1e4, positions=1)
    mg = B.tn_compile(g.tg, None, 1 << 20)
    assert [B.tn_memgraph_vertex(mg, v).bytes for v in range(3)] == [2560, 40, 2560]
    B.tn_memgraph_simulate(mg)
    B.tn_memgraph_destroy(mg)


def test_sizes_past_what_a_launch_counts(g):
    C, R = B.TN_OP_ATTN_COMBINE, B.TN_OP_ATTN_BWD
    rows = 2 ** 25
    part, odd = g.inp(rows, 2 * 64 + 4), g.inp(2 ** 26, 2 * 33 + 4)
    assert g.op(C, [part], rows, 128, head_dim=64, hpg=2, finish=1) >= 0
    _refused(g, C, [odd], 2 ** 26, 66, head_dim=33, hpg=2, finish=1)
    assert g.op(C, [odd], 2 ** 24, 66, head_dim=33, hpg=2, finish=1) >= 0
    do = g.inp(2 ** 27, 2)
    _refused(g, R, [do, do, do], 2 ** 27, 4, mode=4, n_q_tiles=1, n_col_tiles=1, head_dim=1)
