"""The tiler's options on heads and scores on the CPU: the library's taskgraph under the oracle's interpreter against the untiled
decoder, the compiled memgraph under the checkers, and what is refused."""
import numpy as np
import pytest

import heads_cases as C
import util
from oracle import heads_ref as R
from oracle import lora_ref as L
from oracle import llama_ref
from oracle import tiled as T
from paper_2405_16283_amd import binding as B
from paper_2405_16283_amd import harness as H


def _interpreted(cfg, wide, heads, **kw):
    tg = B.tn_build_llama(H.llama_config_struct(cfg, heads=heads, **kw))
    try:
        otg = util.oracle_taskgraph(tg)
        tiles = {v: np.ascontiguousarray(a, dtype=np.float64) for v, a in H.cut_host_tiles(tg, wide).items()}
        vals = T.evaluate(otg, tiles)
        d = cfg.d_model
        return util.assemble_named(otg, vals, "y", cfg.tokens, d), otg
    finally:
        B.tn_taskgraph_destroy(tg)


@pytest.mark.parametrize("options", C.OPTIONS)
@pytest.mark.parametrize("kw", [{}, dict(v_transposed=False, attn_whole_rows=True), dict(weights_transposed=False, fuse_epilogues=3)],
                         ids=["blocks", "whole rows", "fused"])
def test_graphs_compute_the_decoder(options, kw):
    for name in ("ragged_f32", "batch2_f32"):
        cfg, full, wide, heads = C.case(name, options)
        y, _ = _interpreted(cfg, wide, heads, **kw)
        assert llama_ref.rel_err(y, C.exact(cfg, wide, heads)) < 1e-5  # fp32 storage between vertices


@pytest.mark.parametrize("options", [o for o in C.OPTIONS if C.OPTIONS[o].get("score_spans") != 2])
def test_decode_steps_continue_the_sequence(options):
    cfg, full, wide, heads = C.case("decode_f32", options)
    y, _ = _interpreted(cfg, wide, heads)
    assert llama_ref.rel_err(y, C.exact(cfg, wide, heads)) < 1e-5


def test_the_reference_without_options_is_the_plain_one():
    cfg, full, wide, heads = C.case("ragged_f32", "plain", lora=True)
    lora = {k: a for k, a in wide.items() if k.split(".")[0] in ("aq", "bq", "av", "bv")}
    w = {k: a for k, a in wide.items() if k not in lora and k != "probe"}
    y, g = C.exact(cfg, wide, heads, train=True)
    y2, g2 = L.loss_and_grads(cfg, w, lora, wide["x"], wide["probe"])
    assert llama_ref.rel_err(y, y2) < 1e-12
    for k in g:
        assert llama_ref.rel_err(g[k], g2[k]) < 1e-10


def test_without_options_the_graph_is_what_it_was():
    cfg = C.config("ragged_f32")
    for kw in ({}, dict(lora_rank=16, train=True)):
        a, b = (B.tn_build_llama(H.llama_config_struct(cfg, heads=h, **kw)) for h in (None, {}))
        x, y = H.export_taskgraph(a), H.export_taskgraph(b)
        assert x == y and not {"head_rope", "head_rope_bwd"} & set(x["kind"]) and "i32" not in x["dtype"]
        B.tn_taskgraph_destroy(a)
        B.tn_taskgraph_destroy(b)


def test_finished_rows_need_no_combine():
    cfg, full, wide, heads = C.case("batch2_f32", "documents")
    y, tg = _interpreted(cfg, wide, heads, attn_whole_rows=True)
    assert "attn_combine" not in tg.kind and "attn_block" in tg.kind
    y, tg = _interpreted(cfg, wide, {}, attn_whole_rows=True)
    assert "attn_combine" in tg.kind


@pytest.mark.parametrize("options", ["rotations", "documents", "everything", "everything, both sides"])
@pytest.mark.parametrize("train", [False, True])
def test_memgraphs_under_a_cap(options, train):
    cfg, full, wide, heads = C.case("batch2_f32", options, lora=train)
    kw = dict(lora_rank=16, train=True) if train else {}
    tg = B.tn_build_llama(H.llama_config_struct(cfg, heads=heads, **kw))
    mg = B.tn_compile(tg, None, (int(0.6 * H.uncapped_peak(tg)) + 255) // 256 * 256, B.tn_compile_opts(max_lookahead_bytes=B.UINT64_MAX, drop_clean_inputs=1))
    B.tn_memgraph_simulate(mg)
    util.check_all(util.task_preds(tg), util.oracle_memgraph(mg), n_random=2)
    B.tn_memgraph_destroy(mg)
    B.tn_taskgraph_destroy(tg)


def test_refusals():
    cfg = C.config("c1")

    def refused(cfg=cfg, heads=None, **kw):
        with pytest.raises(B.TurnipError) as e:
            B.tn_build_llama(H.llama_config_struct(cfg, heads=heads, **kw))
        assert e.value.message

    narrow = cfg.with_(tile=32, attn_block=32)  # half a head
    for h in (dict(qk_norm=1), dict(rope_half=1), dict(rotary_dim=32), dict(rope_factor=2.0), dict(row_positions=1)):
        refused(narrow, h)
    for h in (dict(rotary_dim=66), dict(rotary_dim=31), dict(rope_factor=2.0, rope_len0=10), dict(rope_factor=2.0, rope_len0=-10), dict(rope_half=1, rope_factor=0.5), dict(rope_factor=0.5), dict(rope_factor=float("nan")),
              dict(score_cap=-1.0), dict(score_cap=1e-9), dict(score_cap=float("nan")), dict(score_spans=3), dict(score_spans=-1)):
        refused(cfg, h)
    for h in (dict(score_cap=1.0), dict(score_slopes=1), dict(score_spans=1)):
        refused(cfg, h, materialize_scores=True)
    refused(C.config("decode_f32"), dict(score_spans=2))


def test_unknown_fields_of_heads_are_refused():
    for wrong in ("scor_cap", "layers", "tile"):
        with pytest.raises(ValueError, match=wrong):
            H.llama_config_struct(C.config("c1"), heads={"score_cap": 1.0, wrong: 1})


@pytest.mark.parametrize("kw", [{}, dict(checkpoint=True)])
def test_training_by_a_rule_takes_its_statistics_from_one_partial(kw):
    """Of finished rows in bf16 they put gradients of rows that see two or three keys up to 1e-2 off."""
    cfg, full, wide, heads = C.case("batch2_f32", "documents", lora=True)
    tg = B.tn_build_llama(H.llama_config_struct(cfg, heads=heads, lora_rank=16, train=True, **kw))
    try:
        x = H.export_taskgraph(tg)
        stats = [v for v, k in enumerate(x["kind"]) if k == "attn_bwd" and x["params"][v]["mode"] == 4]
        assert stats
        for v in stats:
            ins = x["inputs"][v]
            assert x["params"][v]["nk"] == 1 and len(ins) == 2 and x["kind"][ins[0]] == "attn_block" and x["dtype"][ins[0]] == "f32"
            assert x["params"][ins[0]]["k_pos0"] == 0
    finally:
        B.tn_taskgraph_destroy(tg)
