"""Decoders with options on heads and scores on the GPU, through the session: prefill, decode steps and the fine-tuning step, under a cap,
against the untiled decoder (fp32) and the oracle's interpreter of the same graph (bf16)."""
import numpy as np
import pytest

import heads_cases as C
import util
from oracle import llama_ref as R
from oracle import tiled as T
from paper_2405_16283_amd import binding as B
from paper_2405_16283_amd import harness as H

pytestmark = pytest.mark.gpu
OPTS = B.tn_exec_opts(policy=B.TN_POLICY_RANDOM, order_seed=3, max_delay_us=30)


def _orders_agree(s, out):
    for opts in (B.tn_exec_opts(policy=B.TN_POLICY_BY_ORDER, max_batch=1920, queue_depth=3), B.tn_exec_opts(policy=B.TN_POLICY_LIFO, max_batch=1)):
        again, _ = s.run(opts)
        for k in out:
            np.testing.assert_array_equal(again[k], out[k])


def _runs(*forms):
    """Every form with all options that it takes (spans instead of the causal mask do not go with decode steps)."""
    return [pytest.param(n, kw, o, id=f"{n}-{i}-{o}") for i, (n, kw) in enumerate(forms) for o in C.OPTIONS
            if not (n.startswith("decode") and C.OPTIONS[o].get("score_spans") == 2)]


@pytest.mark.parametrize("name,kw,options", _runs(("ragged_f32", {}), ("batch2_f32", dict(v_transposed=False, attn_whole_rows=True)),
                                                  ("decode_f32", dict(v_transposed=False))))
def test_prefill_and_decode_fp32(name, kw, options):
    cfg, full, wide, heads = C.case(name, options)
    s = H.GpuSession(cfg, full, heads=heads, **kw)
    try:
        out, rep = s.run(OPTS)
        assert R.rel_err(out["y"].astype(np.float64), C.exact(cfg, wide, heads)) < 1e-4
        _orders_agree(s, out)
    finally:
        s.close()


@pytest.mark.parametrize("name,kw,options", _runs(("ragged_bf16", dict(v_transposed=False)), ("ragged_bf16", dict(v_transposed=True)),
                                                  ("decode_bf16", dict(v_transposed=False, fuse_epilogues=3))))
def test_prefill_and_decode_bf16(name, kw, options):
    cfg, full, wide, heads = C.case(name, options)
    cfg = cfg.with_(layers=1)  # as the other bf16 graphs: two layers of two correct pipelines drift apart
    s = H.GpuSession(cfg, full, heads=heads, **kw)
    try:
        out, rep = s.run(OPTS)
        otg = util.oracle_taskgraph(s.tg)
        tiles = {v: np.ascontiguousarray(a, dtype=np.float64) for v, a in H.cut_host_tiles(s.tg, wide).items()}
        ref = util.assemble_named(otg, T.evaluate(otg, tiles), "y", cfg.tokens, cfg.d_model)
        assert R.rel_err(C.wide_array(out["y"]), ref) < 2e-2
        _orders_agree(s, out)
    finally:
        s.close()


@pytest.mark.parametrize("options", C.OPTIONS)
@pytest.mark.parametrize("name,kw", [("ragged_f32", {}), ("batch2_f32", dict(v_transposed=False)), ("ragged_bf16", dict(v_transposed=False)),
                                     ("ragged_bf16", dict(v_transposed=False, checkpoint=True)),
                                     ("batch2_f32", dict(recompute_normed=True, recompute_gate_up=True))])
def test_fine_tuning_step(name, kw, options):
    """fp32: 1e-4.  bf16: rounding every stored tensor and gradient, and nothing else, puts the oracle's own gradients up to 4.3e-2 from the exact
    ones (bq.0 of "everything"; 4.03e-2 with spans both ways), so no fixed 4e-2 holds: results are held to 1.5 times what rounding alone does
    to the worst of the case's gradients, as the full-width fine-tuning step is."""
    cfg, full, wide, heads = C.case(name, options, lora=True)
    y, g = C.exact(cfg, wide, heads, train=True)
    tol = 1e-4
    if cfg.dtype == "bf16":
        _, rounded = C.exact(cfg, wide, heads, train=True, storage="bf16")
        tol = 1.5 * max(R.rel_err(rounded[k], g[k]) for k in g)
    s = H.GpuSession(cfg, full, lora_rank=16, train=True, heads=heads, **kw)
    try:
        out, rep = s.run(OPTS)
        errs = {"y": R.rel_err(C.wide_array(out["y"]), y), "dx": R.rel_err(C.wide_array(out["dx"]), g["x"])}
        errs.update({k: R.rel_err(C.wide_array(out["d" + k]), g[k]) for k in g if k != "x"})
        print({k: f"{e:.1e}" for k, e in errs.items()}, flush=True)
        assert max(errs.values()) < tol, errs
        _orders_agree(s, out)
    finally:
        s.close()


def test_inputs_already_in_place_are_not_copied_again():
    """Device-resident inputs that the memgraph gives a place of their own stay there: the second run needs no placing."""
    cfg, full, wide, heads = C.case("batch2_f32", "everything")
    cfg = cfg.with_(weights_resident=True, x_resident=True)
    s = H.GpuSession(cfg, full, cap=64 << 20, heads=heads, compile_opts=B.tn_compile_opts(max_lookahead_bytes=B.UINT64_MAX, next_fit=1))
    try:
        first, _ = s.run(OPTS)
        s.out_slab.fill_(0xFF)
        s.execute(OPTS)
        np.testing.assert_array_equal(s.outputs()["y"], first["y"])
    finally:
        s.close()


def test_arrays_of_other_types_are_converted_or_refused():
    """As before tensors of integers were inputs: what converts without a change of kind does, and nothing is taken for its bytes."""
    cfg, full, wide, heads = C.case("batch2_f32", "everything")
    other = {k: a.astype(np.int64 if a.dtype == np.int32 else np.float64) for k, a in full.items()}
    got = []
    for inputs in (full, other):
        s = H.GpuSession(cfg, inputs, heads=heads)
        try:
            got.append(s.run(OPTS)[0]["y"])
        finally:
            s.close()
    np.testing.assert_array_equal(*got)
    cfg, full, wide, heads = C.case("ragged_bf16", "plain")
    with pytest.raises(TypeError):
        H.GpuSession(cfg, {**full, "x": wide["x"].astype(np.float32)})
