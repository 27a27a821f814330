"""Decoders with options on heads and scores, for the tests of the tiler on the CPU and on the GPU."""
import numpy as np

from oracle import heads_ref as H
from workloads import config, make_llama_inputs, make_lora_inputs, to_bf16_bits

ROTATIONS = dict(qk_norm=1, rope_half=1, rotary_dim=32, rope_factor=4.0, rope_len0=64, rope_low=1.0, rope_high=4.0, row_positions=1)
OPTIONS = {
    "plain": {},
    "normed heads": dict(qk_norm=1),
    "rotations": ROTATIONS,
    "half, scaled": dict(rope_half=1, rope_factor=8.0),
    "capped": dict(score_cap=2.0),
    "slopes": dict(score_slopes=1, score_cap=5.0),
    "documents": dict(score_spans=1, row_positions=1, qk_norm=1, score_cap=3.0),
    "prefix": dict(score_spans=2, score_slopes=1),
    "everything": dict(ROTATIONS, score_cap=3.0, score_slopes=1, score_spans=1),
    "everything, both sides": dict(ROTATIONS, score_cap=3.0, score_slopes=1, score_spans=2),
}


def case(name, options, lora=False, seed=0, padding=9):
    """(config, full arrays in storage type, the same in float64, options)"""
    cfg, heads = config(name), OPTIONS[options]
    full = make_llama_inputs(cfg, seed)
    if lora:
        full.update(make_lora_inputs(cfg, seed, rank=16, b_std=0.02))
    rng = np.random.default_rng(seed + 7)
    seq, tokens = cfg.total_seq, cfg.tokens
    if heads.get("qk_norm"):
        for l in range(cfg.layers):
            for n in ("gq", "gk"):
                g = (1.0 + 0.2 * rng.standard_normal(cfg.head_dim)).astype(np.float32)
                full[f"{n}.{l}"] = g if cfg.dtype == "f32" else to_bf16_bits(g)
    at = np.arange(seq)
    cut = seq // 3
    if heads.get("row_positions"):
        full["positions"] = np.tile(np.where(at < cut, at, at - cut), cfg.batch).astype(np.int32).reshape(-1, 1)
    if heads.get("score_spans") == 1:  # two packed documents; the prefill's last rows are padding that sees nothing
        s = np.where(at[:, None] < cut, [[0, cut]], [[cut, seq]])
        s[cfg.seq - padding:cfg.seq] = 0
        full["spans"] = np.tile(s, (cfg.batch, 1)).astype(np.int32)
    if heads.get("score_spans") == 2:  # a prefix that everybody sees, causal behind it
        full["spans"] = np.tile(np.stack([0 * at, np.maximum(at + 1, cut)], 1), (cfg.batch, 1)).astype(np.int32)
    if heads.get("score_slopes"):
        full["slopes"] = (2.0 ** -(1.0 + np.arange(cfg.n_heads))).astype(np.float32).reshape(1, -1)
    wide = {k: wide_array(a) for k, a in full.items()}
    return cfg, full, wide, heads


def wide_array(a):
    from workloads import bf16_bits_to_f32
    return (bf16_bits_to_f32(a) if a.dtype == np.uint16 else a).astype(np.float64)


def exact(cfg, wide, heads, train=False, storage=None):
    w = {k: a for k, a in wide.items() if k != "probe"}
    return H.decoder(cfg, w, heads, wide["probe"] if train else None, storage)
