"""runner.DeviceTrainer beside the step itself (tests/test_training_step.py): what its buffers do between steps and what it refuses.
"""
import numpy as np
import pytest

from paper_2409_06206_amd import synth

B, H, W, C, HEADS, GROUPS, WINDOW, SHIFT, HIDDEN, LAYERS = 2, 16, 24, 60, 6, 2, 8, 4, 120, 2
EDGES = [1, 2, 4]


def _values(dtype, seed, edges=EDGES):
    """Parameters of the layers, of the norm, and inputs."""
    rng = np.random.default_rng(seed)
    layers = [synth.astl_params(C, HEADS, GROUPS, WINDOW, HIDDEN, 300 + 10 * seed + l, "stress") for l in range(LAYERS)]
    if edges is not None:
        for p in layers:
            del p["table"]
            p["buckets"] = rng.normal(0, 1, ((2 * (len(edges) + 1)) ** 2, HEADS)).astype(np.float32)
    layers = [{k: synth.quantize(v, dtype) for k, v in p.items()} for p in layers]
    norm = [synth.quantize(v.astype(np.float32), dtype) for v in (1 + 0.1 * rng.normal(size=C), 0.1 * rng.normal(size=C))]
    return layers, norm, [synth.quantize(a, dtype) for a in synth.activations(B, H, W, C, 11 + seed)]


def _new(dtype, device="cuda:0", edges=EDGES, **kw):
    from paper_2409_06206_amd import runner
    kw = {**dict(edges=edges, lr=1e-2, weight_decay=0.1, max_norm=0.5, seed=7), **kw}
    return runner.DeviceTrainer(B, H, W, C, HEADS, GROUPS, WINDOW, SHIFT, dtype, HIDDEN, LAYERS, device=device, **kw)


# ---- without a GPU ---------------------------------------------------------------------------------------------------------------

@pytest.fixture
def on_cpu(monkeypatch):
    """The trainer's own bookkeeping, with its buffers in host memory: only the plan needs a GPU."""
    from paper_2409_06206_amd import adamw

    class Plan:
        def __init__(self, tensors, buffer):
            self.tensors, self.buffer = tensors, buffer

    monkeypatch.setattr(adamw, "adamw_plan", lambda desc, tensors, buffer, stream=None: Plan(tensors, buffer))


def test_values_that_do_not_fit_are_refused_and_change_nothing(on_cpu):
    t = _new("f32", "cpu")
    layers, norm, (x, dz) = _values("f32", 0)
    t.set_params(layers, *norm)
    t.set_inputs(x, dz)
    for bad in ((x[:1], dz), (x, dz[:, :8]), (x[..., :1], None)):
        with pytest.raises(ValueError, match="values"):
            t.set_inputs(*bad)
    assert np.array_equal(t.stack.x.numpy(), x) and np.array_equal(t.dz.numpy(), dz)
    t.step.fill_(4)
    other, other_norm, _ = _values("f32", 1)
    short = [dict(p) for p in other]
    del short[1]["w_fc2"]
    wide = [dict(p) for p in other]
    wide[0]["b_fc1"] = np.zeros(2 * HIDDEN, np.float32)
    one = [dict(p) for p in other]
    one[0]["b_fc1"] = np.zeros(1, np.float32)   # (would go to all places)
    for bad in ((short, *other_norm), (wide, *other_norm), (one, *other_norm), (other[:1], *other_norm), (other, other_norm[0][:-1], other_norm[1])):
        with pytest.raises(ValueError):
            t.set_params(*bad)
    assert int(t.step) == 4
    for l, p in enumerate(layers):
        for k, v in p.items():
            assert np.array_equal(t.params[f"{l}.{k}"].numpy(), v), k
