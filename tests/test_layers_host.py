"""Layers' configurations and the optimizer on the host (no GPU)."""
import torch


def test_configuration_by_position():
    """nm, mode, seed, stream_id, reuse_every, precision, step, auto_advance, in this order; what came later stands behind them"""
    from paper_2203_10991_amd.autograd import NMConfig
    cfg = NMConfig("1:2", 1, 2, 3, 4, "q8", 8, True)
    assert (cfg.nm, cfg.mode, cfg.seed, cfg.stream_id, cfg.reuse_every, cfg.precision, cfg.step, cfg.auto_advance) == ("1:2", 1, 2, 3, 4, "q8", 8, True)
    assert cfg.dense == "native" and cfg.current_seed() == 4
