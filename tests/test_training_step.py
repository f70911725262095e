"""A training step of a sequence of whole layers, its operators together as they are used: bucketed bias tables, the layers, a LayerNorm, their
gradients, the norm and AdamW (runner.DeviceTrainer).

Gradients are held against the oracle of the layers at the tolerances of their own tests (1e-5 and 2e-2 of a tensor's largest value); the LayerNorm
adds one more stage of that kind.  The update is held against its definition on the gradients that the kernels gave.
"""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as ops
from paper_2409_06206_amd import synth
from tests import parity

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
B, H, W, C, HEADS, GROUPS, WINDOW, SHIFT, HIDDEN, LAYERS = 2, 16, 24, 60, 6, 2, 8, 4, 120, 2
EDGES = [1, 2, 4]   # 8 buckets an axis: distances 0, 1, 2-3 and 4-7 on either side


def _trainer(dtype, bits=32, edges=EDGES, seed=0, flags=0, every=0):
    from paper_2409_06206_amd import runner
    t = runner.DeviceTrainer(B, H, W, C, HEADS, GROUPS, WINDOW, SHIFT, dtype, HIDDEN, LAYERS, every, flags=flags, edges=edges, lr=1e-2,
                             weight_decay=0.1, max_norm=0.5, state_bits=bits, seed=7)
    rng = np.random.default_rng(seed)
    layers = [synth.astl_params(C, HEADS, GROUPS, WINDOW, HIDDEN, 300 + l, "stress") for l in range(LAYERS)]
    if edges is not None:
        for p in layers:
            del p["table"]
            p["buckets"] = rng.normal(0, 1, ((2 * (len(edges) + 1)) ** 2, HEADS)).astype(np.float32)
    layers = [{k: synth.quantize(v, dtype) for k, v in p.items()} for p in layers]
    norm = [synth.quantize(v.astype(np.float32), dtype) for v in (1 + 0.1 * rng.normal(size=C), 0.1 * rng.normal(size=C))]
    x, dz = (synth.quantize(a, dtype) for a in synth.activations(B, H, W, C, 11))
    t.set_params(layers, *norm)
    t.set_inputs(x, dz)
    return t, layers, norm, x, dz


def _oracle_gradients(layers, norm, x, dz, dtype, edges):
    from oracle import astl_oracle
    at = None if edges is None else ops.window_bucket(WINDOW, edges).numpy()
    full = [{**p, "table": p["buckets"][at]} if edges is not None else p for p in layers]
    for p in full:
        p.pop("buckets", None)
    kw = dict(heads=HEADS, groups=GROUPS, window=WINDOW, shift=SHIFT, store=lambda a: synth.quantize(a, dtype))
    y = synth.quantize(astl_oracle.stack_forward(x, full, **kw), dtype)
    rows = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float64)).reshape(-1, C)  # noqa: E731
    gamma, beta = (torch.from_numpy(np.asarray(v, dtype=np.float64)) for v in norm)
    z, _, _ = ops.lnorm_forward(rows(y), gamma, beta, 1e-5)
    dy, dg, db = ops.lnorm_backward(rows(y), rows(dz), gamma, None, 1e-5)
    dy = synth.quantize(dy.numpy().reshape(B, H, W, C), dtype)
    _, grads = astl_oracle.stack_backward(x, dy, full, **kw)
    out = {"norm_w": dg.numpy(), "norm_b": db.numpy()}
    for l, g in enumerate(grads):
        out.update({f"{l}.{k}": v for k, v in g.items() if edges is None or k != "table"})
        if edges is not None:
            d = np.zeros(((2 * (len(edges) + 1)) ** 2, HEADS))
            np.add.at(d, at, g["table"])
            out[f"{l}.buckets"] = d
    return z.numpy().reshape(B, H, W, C), out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("edges", [EDGES, None])
def test_gradients_of_a_step(dtype, edges):
    t, layers, norm, x, dz = _trainer(dtype, edges=edges)
    t.forward()
    t.backward()
    torch.cuda.synchronize()
    z, want = _oracle_gradients(layers, norm, x, dz, dtype, edges)
    from paper_2409_06206_amd import runner
    errs = {"z": parity.rel_err(runner.to_host(t.z), z)}
    errs.update({k: parity.rel_err(runner.to_host(t.grads[k]), w) for k, w in want.items()})
    assert set(t.grads) == set(want)
    # two layers and a norm: three stages of a layer's tolerance each
    bad = {k: e for k, e in errs.items() if not e <= 3 * parity.TOL[dtype]}
    assert not bad, bad


@pytest.mark.parametrize("dtype,bits", [("f32", 32), ("bf16", 32), ("bf16", 8)])
def test_update_of_a_step(dtype, bits):
    t, *_ = _trainer(dtype, bits)
    t.forward()
    t.backward()
    held = t.masters or t.params
    before = {k: v.double().cpu() for k, v in held.items()}
    t.update()
    torch.cuda.synchronize()
    grads = {k: v.double().cpu() for k, v in t.grads.items()}
    norm = float(torch.sqrt(sum((g ** 2).sum() for g in grads.values())))
    assert abs(float(t.grad_norm) - norm) <= 2 * U * norm and norm > 0.5 and int(t.step) == 1
    for k, p in before.items():
        wd = 0.1 if k.split(".")[-1] in t.DECAYED else 0.0
        g = grads[k]
        p1, m1, v1 = ops.adamw_update(p, g, torch.zeros_like(p), torch.zeros_like(p), 1, 1e-2, 0.9, 0.999, 1e-8, wd, 0.5 / norm)
        # first step from zeros: an update of about lr, its error 16 u of it twice (see the operator's own tests)
        assert ((held[k].double().cpu() - p1).abs() <= 4 * U * p.abs() + 64 * U * 1e-2 + U * p1.abs()).all(), k
        if dtype == "bf16":
            assert torch.equal(t.params[k], t.masters[k].to(torch.bfloat16)), k


@pytest.mark.parametrize("dtype,bits,every", [("f32", 32, 0), ("bf16", 8, 0), ("bf16", 32, 1)])
def test_steps_replayed_from_a_graph_are_the_eager_ones(dtype, bits, every):
    """Five steps on changing inputs: one set of buffers eagerly, one by a captured step; the same bits throughout."""
    from paper_2409_06206_amd import gswa, runner
    eager, *_ = _trainer(dtype, bits, flags=gswa.GSWA_DETERMINISTIC, every=every)
    replayed, *_ = _trainer(dtype, bits, flags=gswa.GSWA_DETERMINISTIC, every=every)

    def one(t):
        t.forward()
        t.backward()
        t.update()

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        one(replayed)
    # parameter gradients of part of the layers' path are summed by atomics: the graph takes the eager step's, bit for bit, where they differ
    for n in range(5):
        x, dz = (runner.to_device(synth.quantize(a, dtype), dtype) for a in synth.activations(B, H, W, C, 50 + n))
        for t in (eager, replayed):
            t.stack.x.copy_(x)
            t.dz.copy_(dz)
        graph.replay()
        one(eager)
        torch.cuda.synchronize()
        assert torch.equal(eager.z, replayed.z), n
        for k in eager.grads:
            a, b = eager.grads[k].double(), replayed.grads[k].double()
            assert float((a - b).abs().max()) <= 1e-5 * float(a.abs().max()) + 1e-30, (n, k)
        assert int(replayed.step) == int(eager.step) == n + 1
        for k, p in eager.params.items():   # the next step starts from the same parameters and states
            assert float((p.double() - replayed.params[k].double()).abs().max()) <= 0.05, (n, k)
            replayed.params[k].copy_(p)
            if eager.masters:
                replayed.masters[k].copy_(eager.masters[k])
            for s in eager.states[k]:
                replayed.states[k][s].copy_(eager.states[k][s])


def test_steps_on_two_streams():
    """Two trainings at once, each on a stream of its own, are those run one after the other."""
    sets = [[_trainer("f32", seed=n)[0] for n in range(2)] for _ in range(2)]

    def steps(t, stream=None):
        for _ in range(3):
            t.forward(stream)
            t.backward(stream)
            t.update(stream)

    for t in sets[0]:
        steps(t)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for t, s in zip(sets[1], streams):
        steps(t, s)
    torch.cuda.synchronize()
    for a, b in zip(*sets):
        for k in a.params:
            assert torch.equal(a.params[k], b.params[k]), k


def test_new_parameters_start_over():
    t, layers, norm, _, _ = _trainer("bf16", 8)
    t.forward()
    t.backward()
    ends = []
    for _ in range(2):
        for _ in range(3):
            t.update()   # (on the same gradients: those of the layers are not the same bits every run)
        assert int(t.step) == 3
        ends.append({k: v.clone() for k, v in t.params.items()})
        t.set_params(layers, *norm)
        assert int(t.step) == 0
    for k, v in ends[0].items():
        assert torch.equal(v, ends[1][k]), k


def test_gradients_added_up_over_steps_are_refused():
    from paper_2409_06206_amd import gswa
    with pytest.raises(ValueError, match="ACCUM"):
        _trainer("f32", flags=gswa.GSWA_ACCUM_WGRAD)
