"""Layers' configurations and the optimizer on the host (no GPU)."""
import torch


def test_configuration_by_position():
    """nm, mode, seed, stream_id, reuse_every, precision, step, auto_advance, in this order; what came later stands behind them"""
    from paper_2203_10991_amd.autograd import NMConfig
    cfg = NMConfig("1:2", 1, 2, 3, 4, "q8", 8, True)
    assert (cfg.nm, cfg.mode, cfg.seed, cfg.stream_id, cfg.reuse_every, cfg.precision, cfg.step, cfg.auto_advance) == ("1:2", 1, 2, 3, 4, "q8", 8, True)
    assert cfg.dense == "native" and cfg.current_seed() == 4


def test_optimizer_copied_and_pickled():
    """(a file of this test's own; plain pickle has no way for e4m3 tensors in this torch.)  A copy keeps how the states are held, the masters and the seed beside what torch's own state has"""
    import copy
    import io

    from paper_2203_10991_amd.optim import NMAdamW
    p = torch.nn.Parameter(torch.ones(300, dtype=torch.bfloat16))
    opt = NMAdamW([p], lr=0.5, states="q8", master=True, seed=7)
    opt._state(p)
    file = io.BytesIO()
    torch.save(opt, file)
    file.seek(0)
    for other in (copy.deepcopy(opt), torch.load(file, weights_only=False)):
        assert (other.states, other.master, other.seed, other.defaults["lr"]) == ("q8", True, 7, 0.5)
        q, = other.param_groups[0]["params"]
        assert q is not p and other._state(q).keys() == opt.state[p].keys() and other._state(q)["exp_avg"].dtype == torch.float8_e4m3fn
        fresh = torch.nn.Parameter(torch.ones(5, dtype=torch.bfloat16))
        other.add_param_group({"params": [fresh]})
        assert "master" in other._state(fresh)


def test_a_step_that_fails_is_not_counted():
    import pytest

    from paper_2203_10991_amd.optim import NMAdamW
    good, bad = torch.nn.Parameter(torch.ones(4)), torch.nn.Parameter(torch.ones(4, dtype=torch.float16))
    for p in (good, bad):
        p.grad = torch.ones_like(p)
        opt = NMAdamW([p])
        for _ in range(2):
            with pytest.raises((ValueError, TypeError)):             # not on the GPU, not a type it takes
                opt.step()
        assert opt.state[p]["step"] == 0 and bool((p == 1).all())


def test_convolution_knows_the_dense_products():
    """A convolution's dense products are torch's whatever linear layers of the same configuration take; a value that no layer knows is refused, as linear layers do"""
    import pytest

    from paper_2203_10991_amd.autograd import NMConfig, NMConv2d
    x = torch.randn(2, 8, 5, 5)
    layer = NMConv2d(8, 16, 3, padding=1, cfg=NMConfig(dense="i8"))
    assert torch.equal(layer(x), torch.nn.functional.conv2d(x, layer.weight, layer.bias, padding=1))
    layer.cfg.dense = "i4"
    with pytest.raises(ValueError, match="dense"):
        layer(x)


def test_self_attention_built_on_the_meta_device():
    """frequencies are values, not a shape; rotary_freqs itself goes to the default device as torch's own factories do, and what a call under inference_mode makes can be saved for a gradient"""
    import paper_2203_10991_amd as nm
    from paper_2203_10991_amd.autograd import NMSelfAttention
    with torch.device("meta"):
        layer = NMSelfAttention(64, 4, rotary_options={"base": 500.0})
        assert nm.rotary_freqs(16, device="cpu").device.type == "cpu" and nm.rotary_freqs(16).is_meta
    layer = layer.to_empty(device="cpu")
    assert layer.qkv.weight.device.type == "cpu" and torch.equal(layer._frequencies(torch.device("cpu")), nm.rotary_freqs(16, 500.0))
    with torch.inference_mode():
        assert not nm.rotary_freqs(16).is_inference() and not NMSelfAttention(64, 4)._freqs.is_inference()
