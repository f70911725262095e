"""AdamW over many tensors (adamw.h) against its definition in 64 bits, and what its entry points refuse.

Tolerances, u = 2^-24 (half a step of fp32, relative).  The clipping factor is off by at most 3 u (the norm's rounding, a quotient), so
|err m'| <= 3 u beta1 |m| + 6 u (1 - beta1) |g| (rounded factors, product, sum) <= 8 u (beta1 |m| + (1 - beta1) |g|) =: 8 u M;
|err v'| <= 12 u v' (g enters squared; no cancellation).  The update d = rate m' / (sqrt(v') / root + eps): |err d| <= 16 u (|d| + rate M / (sqrt(v') / root + eps)).
|err p'| <= 4 u |p| + that + u |p'|; a bf16 copy adds 2^-8 |p'|.
8-bit states: what is held has to be a value that the rounding gives within that distance of the exact state: rounding is monotone, so between the
roundings of the two ends.  The same for a bf16 parameter without an fp32 copy.
"""
import ctypes
import math

import pytest
import torch

from oracle import operators_oracle as oracle
from paper_2409_06206_amd import adamw, gswa
from tests.test_abi_cpu import declared_functions

U = 2.0 ** -24
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
gpu = pytest.mark.gpu


# ---- without a GPU ---------------------------------------------------------------------------------------------------------------

def test_exports():
    assert set(declared_functions("adamw.h", "adamw")) == set(adamw.EXPORTS)
    for n in adamw.EXPORTS:
        assert hasattr(adamw.lib(), n)


@pytest.mark.parametrize("change", [dict(state_bits=(1 << 32) + 8), dict(flags=1 << 32)])
def test_numbers_that_a_field_cannot_hold_are_refused(change):
    with pytest.raises(ValueError, match="hold"):
        adamw.make_desc(**change)


def test_seeds_are_taken_modulo_2_to_64():
    assert adamw.make_desc(seed=-1).seed == adamw.make_desc(seed=(1 << 64) - 1).seed == adamw.make_desc(seed=(1 << 65) - 1).seed == (1 << 64) - 1


def _c_tensors(*parts):
    out = (adamw.adamw_tensor * len(parts))()
    for i, p in enumerate(parts):
        out[i] = adamw.adamw_tensor(**p)
    return out


BASE = 1 << 30   # addresses that are never dereferenced: the calls are refused first
STEP = 1 << 20


def _part(i=0, **change):
    at = BASE + i * 16 * STEP
    return {**dict(n=1000, p_dtype=0, g_dtype=0, weight_decay=0.0, p=at, g=at + STEP, m=at + 2 * STEP, v=at + 3 * STEP), **change}


def _plan(desc, parts, buffer=BASE - 256 * STEP):
    plan = adamw.adamw_plan_t()
    return adamw.lib().adamw_plan(ctypes.byref(desc), _c_tensors(*parts), len(parts), buffer, ctypes.byref(plan), None)


@pytest.mark.parametrize("change", [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=2.0 ** -127),
                                    dict(state_bits=16), dict(flags=2)])
def test_bad_descriptors(change):
    n = ctypes.c_size_t()
    assert adamw.lib().adamw_query_bytes(ctypes.byref(adamw.make_desc(**change)), _c_tensors(_part()), 1, ctypes.byref(n)) == gswa.GSWA_EINVAL


@pytest.mark.parametrize("change", [
    dict(n=-1), dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(p_dtype=2), dict(g_dtype=-1), dict(weight_decay=-1.0),
    dict(weight_decay=float("nan")), dict(master=BASE + 4 * STEP), dict(m_exp=BASE + 5 * STEP), dict(p=BASE + 8), dict(g=BASE + STEP + 4),
    dict(g=BASE + 16), dict(m=BASE + 3 * STEP - 16), dict(v=BASE), dict(v=BASE + 2 * STEP + 3984),
])
def test_bad_tensors_are_refused_before_a_launch(change):
    assert _plan(adamw.make_desc(), [_part(1), _part(0, **change)]) == gswa.GSWA_EINVAL


def test_bad_lists_and_buffers():
    L, d, n = adamw.lib(), adamw.make_desc(), ctypes.c_size_t()
    assert L.adamw_query_bytes(ctypes.byref(d), _c_tensors(_part()), 0, ctypes.byref(n)) == gswa.GSWA_EINVAL
    assert L.adamw_query_bytes(ctypes.byref(d), None, 1, ctypes.byref(n)) == gswa.GSWA_EINVAL
    assert L.adamw_query_bytes(ctypes.byref(d), _c_tensors(_part(n=1 << 41)), 1, ctypes.byref(n)) == gswa.GSWA_EUNSUPPORTED
    assert _plan(d, [_part()], BASE - 256 * STEP + 16) == gswa.GSWA_EINVAL
    assert _plan(d, [_part()], BASE + 2 * STEP) == gswa.GSWA_EINVAL          # the buffer over a state
    assert _plan(d, [_part(), _part()]) == gswa.GSWA_EINVAL                  # the same tensor twice
    assert _plan(d, [_part(), _part(1, p=BASE + STEP)]) == gswa.GSWA_EINVAL  # a parameter over another one's gradient
    eight = adamw.make_desc(state_bits=8)
    assert _plan(eight, [_part()]) == gswa.GSWA_EINVAL                       # no exponents
    assert _plan(eight, [_part(m_exp=BASE + 4 * STEP, v_exp=BASE + 4 * STEP + 3)]) == gswa.GSWA_EINVAL   # 4 bytes each


def test_calls_without_a_plan():
    L, p = adamw.lib(), adamw.adamw_plan_t()
    assert L.adamw_norm(ctypes.byref(p), BASE, None) == gswa.GSWA_EINVAL
    assert L.adamw_step(ctypes.byref(p), BASE, 1e-3, None, None, 0.0, None) == gswa.GSWA_EINVAL
    assert L.adamw_unpack(ctypes.byref(p), BASE, None, None) == gswa.GSWA_EINVAL
    assert L.adamw_step(None, BASE, 1e-3, None, None, 0.0, None) == gswa.GSWA_EINVAL


def test_plan_buffers_hold_a_line_per_tensor():
    sizes = []
    for n in (1, 2, 500):
        t = _c_tensors(*[_part(i) for i in range(n)])
        b = ctypes.c_size_t()
        assert adamw.lib().adamw_query_bytes(ctypes.byref(adamw.make_desc()), t, n, ctypes.byref(b)) == 0
        assert b.value % 256 == 0
        sizes.append(b.value)
    assert sizes[0] <= sizes[1] < sizes[2]


def test_tensors_are_checked():
    p = torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        adamw.adamw_plan(adamw.make_desc(), [dict(p=p, g=p, m=p, v=p)], None)
    with pytest.raises(ValueError, match="unknown"):
        adamw.adamw_plan(adamw.make_desc(), [dict(p=p, g=p, m=p, v=p, q=p)], None)
    with pytest.raises(ValueError, match="gradients"):
        adamw.adamw_plan(adamw.make_desc(), [dict(p=p, g=p[:3], m=p, v=p)], None)


def test_the_oracles_rounding_is_right_on_average_and_its_format_holds_what_it_rounds_to():
    x = torch.full((1 << 18,), 1.03)
    r = oracle.round_randomly(x, 3, oracle.noise(5, 1, 0, x.numel())[0])
    assert set(r.unique().tolist()) == {1.0, 1.125}
    assert abs(float(r.mean()) - 1.03) < 5 * 0.125 * math.sqrt(0.24 * 0.76 / x.numel()) + 2.0 ** -16
    a, b, c = oracle.noise(5, 1, 0, 1 << 16), oracle.noise(5, 2, 0, 1 << 16), oracle.noise(6, 1, 0, 1 << 16)
    for i in range(3):
        for other in (a[(i + 1) % 3], b[i], c[i]):   # of other uses, steps and seeds: not correlated
            assert abs(float(torch.corrcoef(torch.stack([a[i].double(), other.double()]))[0, 1])) < 5 / 256


# ---- on the GPU --------------------------------------------------------------------------------------------------------------------

SIZES = [1, 3, 60, 255, 256, 257, 1024, 1350, 2047, 2048, 2049, 7200, 0, 70001]


def _make(sizes, p, g, bits, seed, fresh=False):
    """Lists of parts on the CPU: fp32 values of everything, states of 8 bits as random codes."""
    gen = torch.Generator().manual_seed(seed)
    parts = []
    for i, n in enumerate(sizes):
        level = 10.0 ** torch.randn(1, generator=gen)
        part = dict(p=torch.randn(n, generator=gen) * 0.1, g=torch.randn(n, generator=gen) * level, weight_decay=0.1 * (i % 2))
        if p == "bf16+f32":
            part["master"] = part["p"].clone()
        part["p"] = part["p"].to(TYPE[p[:4]] if p != "f32" else torch.float32)
        part["g"] = part["g"].to(TYPE[g])
        blocks = -(-n // 256)
        if bits == 32:
            part["m"] = torch.randn(n, generator=gen) * level * 0.5 * (not fresh)
            part["v"] = torch.rand(n, generator=gen) * level ** 2 * (not fresh)
        else:
            part["m"], part["v"] = (torch.randint(0, 256, (n,), generator=gen, dtype=torch.uint8) * (not fresh) for _ in range(2))
            part["m_exp"] = torch.randint(110, 130, (blocks,), generator=gen, dtype=torch.uint8) * (not fresh)
            part["v_exp"] = torch.randint(100, 130, (blocks,), generator=gen, dtype=torch.uint8) * (not fresh)
            if not fresh:   # a negative nothing is not a code
                part["m"][part["m"] == 128] = 0
        parts.append(part)
    return parts


def _device(parts):
    return [{k: v.cuda() if torch.is_tensor(v) else v for k, v in part.items()} for part in parts]


def _planned(desc, parts):
    buffer = torch.full((adamw.adamw_query_bytes(desc, parts),), 0x5A, dtype=torch.uint8, device="cuda")
    return adamw.adamw_plan(desc, parts, buffer)


def _between(got, lo, hi, what):
    got = got.double()
    lo, hi = torch.minimum(lo, hi), torch.maximum(lo, hi)
    ok = ((got >= lo) & (got <= hi)) | (torch.isnan(got) & torch.isnan(lo))
    assert bool(ok.all()), (what, int((~ok).sum()), got[~ok][:4], lo[~ok][:4], hi[~ok][:4])


def _check_step(before, after, desc, t, lr, clip):
    """Every tensor of one step, from CPU copies before and after it."""
    first = 0
    for i, (b, a) in enumerate(zip(before, after)):
        n = b["p"].numel()
        eight = desc.state_bits == 8
        m = oracle.held_value(b["m"], b["m_exp"], False) if eight else b["m"]
        v = oracle.held_value(b["v"], b["v_exp"], True) if eight else b["v"]
        master = b.get("master")
        p0 = b["p"] if master is None else master
        wd = b["weight_decay"]
        p1, m1, v1 = oracle.adamw_update(p0, b["g"], m, v, t, lr, desc.beta1, desc.beta2, desc.eps, wd, clip)
        M = desc.beta1 * m.double().abs() + (1 - desc.beta1) * (b["g"].double() * clip).abs()
        em, ev = 8 * U * M, 12 * U * v1
        size = lr / (1 - desc.beta1 ** t) / (torch.sqrt(v1 / (1 - desc.beta2 ** t)) + desc.eps)
        ep = 4 * U * p0.double().abs() + 16 * U * size * (m1.abs() + M) + U * p1.abs()
        n_m, n_v, n_p = oracle.noise(desc.seed, t, first, n)
        if master is not None:
            assert bool(((a["master"].double() - p1).abs() <= ep).all()), ("master", i)
            assert torch.equal(a["p"], a["master"].to(torch.bfloat16)), ("copy", i)
        elif b["p"].dtype == torch.bfloat16:
            _between(a["p"], oracle.round_randomly(p1 - ep, 7, n_p), oracle.round_randomly(p1 + ep, 7, n_p), ("p", i))
        else:
            assert bool(((a["p"].double() - p1).abs() <= ep).all()), ("p", i)
        if eight:
            for k, x, e, noise16, second in (("m", m1, em, n_m, False), ("v", v1, ev, n_v, True)):
                got = oracle.held_value(a[k], a[k + "_exp"], second)
                _between(got, oracle.hold(x - e, noise16, second), oracle.hold(x + e, noise16, second), (k, i))
        else:
            assert bool(((a["m"].double() - m1).abs() <= em).all()), ("m", i)
            assert bool(((a["v"].double() - v1).abs() <= ev).all()), ("v", i)
        first += -(-n // 256) * 256


def _cpu(parts):
    return [{k: v.detach().cpu().clone() if torch.is_tensor(v) else v for k, v in part.items()} for part in parts]


KINDS = [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16"), ("bf16+f32", "f32"), ("bf16+f32", "bf16")]


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p,g", KINDS)
def test_steps(p, g, bits):
    """Three steps, clipped and not, from states of all kinds; nothing is written behind a tensor's end."""
    desc = adamw.make_desc(0.9, 0.999, 1e-8, bits, seed=0x123456789ABCDEF)
    parts = _device(_make(SIZES, p, g, bits, 1))
    guard = []
    for part in parts:   # every array inside a larger one
        for k in ("p", "master", "m", "v", "m_exp", "v_exp"):
            if k in part:
                t = part[k]
                wide = torch.empty(t.numel() + 64, dtype=t.dtype, device="cuda")
                wide.view(torch.uint8).fill_(0xA5)
                wide[: t.numel()] = t
                part[k] = wide[: t.numel()]
                guard.append((wide, t.numel()))
    plan, step, norm = _planned(desc, parts), torch.tensor([6], device="cuda"), torch.zeros(1, device="cuda")
    for n in range(3):
        before = _cpu(parts)
        adamw.adamw_norm(plan, norm)
        most = (0.0, float(norm) / 2, float(norm) * 2)[n]
        adamw.adamw_step(plan, step, 1e-2, norm=norm, max_norm=most)
        torch.cuda.synchronize()
        want = math.sqrt(sum(float(b["g"].double().square().sum()) for b in before))
        assert abs(float(norm) - want) <= 2 * U * want
        _check_step(before, _cpu(parts), desc, 7 + n, 1e-2, most / want if n == 1 else 1.0)
        assert int(step) == 7 + n
    for wide, n in guard:
        assert bool((wide[n:].view(torch.uint8) == 0xA5).all())


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_the_first_step_from_zeros_and_a_late_one(bits):
    for t in (0, 1, 999, 123456789, (1 << 32) + 5):
        desc = adamw.make_desc(0.9, 0.999, 1e-8, bits, seed=t)
        parts = _device(_make([300, 5000], "bf16", "f32", bits, 2, fresh=True))
        plan, step = _planned(desc, parts), torch.tensor([t], device="cuda")
        before = _cpu(parts)
        adamw.adamw_step(plan, step, 1e-3)
        _check_step(before, _cpu(parts), desc, t + 1, 1e-3, 1.0)
        assert int(step) == t + 1


@gpu
@pytest.mark.parametrize("beta1,beta2,eps", [(0.0, 0.0, 0.0), (0.0, 0.99, 1e-6), (0.95, 0.9999, 1e-12)])
def test_other_coefficients(beta1, beta2, eps):
    for bits in (32, 8):
        desc = adamw.make_desc(beta1, beta2, eps, bits, seed=3)
        parts = _device(_make([700], "f32", "f32", bits, 3))
        plan, step = _planned(desc, parts), torch.tensor([2], device="cuda")
        before = _cpu(parts)
        adamw.adamw_step(plan, step, 0.5)
        _check_step(before, _cpu(parts), desc, 3, 0.5, 1.0)


@gpu
def test_types_mixed_in_one_list():
    parts = []
    for i, (p, g) in enumerate(KINDS * 15):   # more tensors than one launch lays out
        parts += _make([17 * i + 5], p, g, 8, 40 + i)
    parts = _device(parts)
    desc = adamw.make_desc(state_bits=8, seed=9)
    plan, step = _planned(desc, parts), torch.tensor([10], device="cuda")
    before = _cpu(parts)
    adamw.adamw_step(plan, step, 1e-3)
    _check_step(before, _cpu(parts), desc, 11, 1e-3, 1.0)


@gpu
def test_learning_rate_on_the_device():
    made = _make([1000, 3000], "f32", "f32", 32, 5)
    a, b = _device(made), _device(made)
    desc, scale = adamw.make_desc(), torch.tensor([0.25], device="cuda")
    adamw.adamw_step(_planned(desc, a), torch.tensor([3], device="cuda"), 1e-2, lr_scale=scale)
    adamw.adamw_step(_planned(desc, b), torch.tensor([3], device="cuda"), 0.25e-2)
    for x, y in zip(a, b):
        assert bool(((x["p"] - y["p"]).abs() <= 4 * U * (y["p"].abs() + 0.01)).all())


@gpu
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_gradients_that_are_not_finite(bad):
    for bits in (32, 8):
        desc = adamw.make_desc(state_bits=bits, flags=adamw.ADAMW_SKIP_NONFINITE)
        made = _make([600, 900], "bf16+f32", "f32", bits, 6)
        made[1]["g"][300] = bad
        parts = _device(made)
        plan, step, norm = _planned(desc, parts), torch.tensor([4], device="cuda"), torch.zeros(1, device="cuda")
        adamw.adamw_norm(plan, norm)
        assert not math.isfinite(float(norm))
        adamw.adamw_step(plan, step, 1e-2, norm=norm, max_norm=1.0)
        assert int(step) == 4
        for x, y in zip(_cpu(parts), made):
            for k in set(x) - {"g", "weight_decay"}:
                assert torch.equal(x[k], y[k]), k
        with pytest.raises(gswa.GswaError):
            adamw.adamw_step(plan, step, 1e-2)   # nothing to go by
        # without the flag and without clipping it stays in its element, in 8 bits in its block's states
        free = adamw.make_desc(state_bits=bits)
        adamw.adamw_step(_planned(free, parts), step, 1e-2)
        after = _cpu(parts)
        assert bool(torch.isfinite(after[0]["master"]).all())
        hit = ~torch.isfinite(after[1]["master"])
        assert int(hit.sum()) == 1 and bool(hit[300])   # (of an infinity too: the update divides it by one)
        if bits == 8:
            m = oracle.held_value(after[1]["m"], after[1]["m_exp"], False)
            assert bool(torch.isnan(m[256:512]).all()) and bool(torch.isfinite(m[:256]).all()) and bool(torch.isfinite(m[512:]).all())
            assert not bool(torch.isnan(oracle.held_value(after[0]["v"], after[0]["v_exp"], True)).any())


@gpu
def test_small_and_large_magnitudes_in_8_bits():
    """Second moments from the smallest number fp32 has to near its largest; a block of zeros; one value far above the others."""
    desc = adamw.make_desc(0.9, 0.999, 1e-30, 8, seed=11)
    n = 256 * 6
    g = torch.zeros(n)
    g[256:512] = torch.logspace(-19, -22, 256)      # squares at the lower end
    g[512:768] = torch.logspace(17, 18, 256)
    g[768:1024] = 1e-6
    g[800] = 1e3
    g[1024:1280] = 1e-45
    g[1300] = -3.0
    z = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")  # noqa: E731
    part = dict(p=torch.zeros(n, device="cuda"), g=g.cuda(), m=z(n), v=z(n), m_exp=z(6), v_exp=z(6))
    plan = _planned(desc, [part])
    adamw.adamw_step(plan, torch.zeros(1, dtype=torch.int64, device="cuda"), 1e-3)
    after = _cpu([part])[0]
    m, v = oracle.held_value(after["m"], after["m_exp"], False), oracle.held_value(after["v"], after["v_exp"], True)
    assert bool((m[:256] == 0).all()) and bool((v[:256] == 0).all())
    for at in (slice(256, 320), slice(512, 768), slice(1300, 1301), slice(800, 801)):
        want = g.double()[at] * 0.1
        assert bool(((m[at] - want).abs() <= want.abs() / 7.99).all())
    want = (g.double() ** 2 * 1e-3)[512:768]
    assert bool(((v[512:768] - want).abs() <= want / 7.99).all())
    assert bool((v[768:800] > 0).all()) and bool((m[768:800] == 0).all())   # 30 powers of two below the block's largest
    assert bool(torch.isfinite(after["p"]).all())


@gpu
def test_what_changes_by_less_than_half_a_step_still_moves():
    """64 steps of decay of a second moment by a thousandth each, and of a bf16 parameter by a 40th of its step: 4096 elements follow the
    formula on average, within 6 deviations of the random roundings."""
    n, steps = 4096, 64
    z = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")  # noqa: E731
    part = dict(p=torch.ones(n, dtype=torch.bfloat16, device="cuda"), g=torch.zeros(n, device="cuda"), m=z(n), v=z(n), m_exp=z(16), v_exp=z(16),
                weight_decay=0.1)
    part["v"].fill_(255 - 8), part["v_exp"].fill_(127)   # code `top` - 8: 2^0
    plan, step = _planned(adamw.make_desc(state_bits=8, seed=21), [part]), torch.zeros(1, dtype=torch.int64, device="cuda")
    for _ in range(steps):
        adamw.adamw_step(plan, step, 1e-3)
    v = oracle.held_value(part["v"].cpu(), part["v_exp"].cpu(), True)
    # a step of v is at most 2^-3 of it: each rounding's variance at most remainder * step <= 0.001 * 0.125, relative
    assert abs(float(v.mean()) - 0.999 ** steps) <= 6 * math.sqrt(steps * 0.001 * 0.125 / n) + steps * 2.0 ** -19
    # of p below 1: 2^-8 a step
    assert abs(float(part["p"].double().mean()) - (1 - 1e-4) ** steps) <= 6 * math.sqrt(steps * 1e-4 * 2.0 ** -8 / n) + steps * 2.0 ** -24


@gpu
def test_unpacked_states():
    desc = adamw.make_desc(state_bits=8)
    made = _make([1, 300, 0, 2048, 5000], "f32", "f32", 8, 8)
    made[1]["m_exp"][1] = 255
    parts = _device(made)
    plan = _planned(desc, parts)
    m, v = (torch.full((plan.elements,), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    adamw.adamw_unpack(plan, m, v)
    at = 0
    for part in made:
        n = part["p"].numel()
        for out, k, second in ((m, "m", False), (v, "v", True)):
            want = oracle.held_value(part[k], part[k + "_exp"], second)
            got = out[at: at + n].double().cpu()
            assert torch.equal(got.nan_to_num(nan=123.0), want.nan_to_num(nan=123.0))
            assert bool((out[at + n: at + -(-n // 256) * 256] == 0).all())
        at += -(-n // 256) * 256
    assert at == plan.elements
    m2 = torch.empty_like(m)
    adamw.adamw_unpack(plan, m2, None)
    assert torch.equal(m.nan_to_num(nan=1.0), m2.nan_to_num(nan=1.0))
    with pytest.raises(gswa.GswaError):
        adamw.adamw_unpack(_planned(adamw.make_desc(), _device(_make([5], "f32", "f32", 32, 1))), m, v)


@gpu
def test_the_same_bits_every_run_and_in_a_replayed_graph():
    made = _make(SIZES + [333] * 50, "bf16", "f32", 8, 12)
    desc = adamw.make_desc(state_bits=8, seed=77)
    sets = []
    for _ in range(3):
        parts = _device(made)
        sets.append((parts, _planned(desc, parts), torch.tensor([0], device="cuda"), torch.zeros(1, device="cuda")))

    def run(s, stream=None):
        adamw.adamw_norm(s[1], s[3], stream)
        adamw.adamw_step(s[1], s[2], 1e-2, norm=s[3], max_norm=5.0, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(sets[2])
    for k in range(4):
        for s in sets:
            for i, part in enumerate(s[0]):
                part["g"].copy_(torch.randn(part["g"].shape, generator=torch.Generator().manual_seed(1000 * k + i)))
        torch.cuda.synchronize()
        run(sets[0])
        run(sets[1], side)
        graph.replay()
        torch.cuda.synchronize()
        for other in sets[1:]:
            assert int(other[2]) == int(sets[0][2]) == k + 1 and torch.equal(other[3], sets[0][3])
            for x, y in zip(sets[0][0], other[0]):
                for name in ("p", "m", "v", "m_exp", "v_exp"):
                    assert torch.equal(x[name], y[name]), (k, name)


@gpu
def test_a_plan_of_empty_tensors():
    e = torch.empty(0, device="cuda")
    plan = _planned(adamw.make_desc(), [dict(p=e, g=e, m=e, v=e)])
    step, norm = torch.tensor([1], device="cuda"), torch.ones(1, device="cuda")
    adamw.adamw_norm(plan, norm)
    adamw.adamw_step(plan, step, 1e-3, norm=norm, max_norm=1.0)
    assert float(norm) == 0 and int(step) == 2


@gpu
@pytest.mark.parametrize("chunks", [1, 2, 63, 64, 65, 200, 1500])
def test_norms_of_few_and_of_many_pieces(chunks):
    """Added by the last workgroup or by a launch of its own: right, the same bits every run, replayed, and in turn with steps, which count on the same counters."""
    made = _make([1024] * (chunks - 1) + [777], "f32", "f32", 32, chunks)
    parts = _device(made)
    plan, norm, step = _planned(adamw.make_desc(), parts), torch.zeros(1, device="cuda"), torch.tensor([0], device="cuda")
    assert plan.c_plan.chunks == chunks
    graph, replayed = torch.cuda.CUDAGraph(), torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        adamw.adamw_norm(plan, replayed)
    for k in range(4):
        for i, part in enumerate(parts):
            part["g"].copy_(made[i]["g"] * (k + 1))
        want = (k + 1) * math.sqrt(sum(float(b["g"].double().square().sum()) for b in made))
        adamw.adamw_norm(plan, norm)
        graph.replay()
        adamw.adamw_step(plan, step, 0.0)
        torch.cuda.synchronize()
        assert abs(float(norm) - want) <= 4 * U * want and torch.equal(norm, replayed) and int(step) == k + 1   # (g (k + 1) is rounded: 2 U more)


@gpu
def test_scalars_inside_the_plans_memory_are_refused():
    parts = _device(_make([500], "f32", "f32", 32, 15))
    plan, at = _planned(adamw.make_desc(), parts), None
    step, norm = torch.tensor([4], device="cuda"), torch.ones(1, device="cuda")
    at = plan.buffer.data_ptr()
    before = plan.buffer.clone(), _cpu(parts)
    for call in (lambda: adamw.adamw_norm(plan, at), lambda: adamw.adamw_step(plan, at + plan.buffer.numel() - 8, 1e-2),
                 lambda: adamw.adamw_step(plan, step, 1e-2, norm=at, max_norm=1.0), lambda: adamw.adamw_step(plan, step, 1e-2, lr_scale=at),
                 lambda: adamw.adamw_step(plan, step, 1e-2, norm=step.data_ptr() + 4, max_norm=1.0)):
        with pytest.raises(gswa.GswaError):
            call()
    adamw.adamw_norm(plan, norm)
    torch.cuda.synchronize()
    assert int(step) == 4 and torch.equal(parts[0]["p"].cpu(), before[1][0]["p"])


@gpu
@pytest.mark.parametrize("sizes", [[1], [700], [4096], [1024] * 70], ids=str)
def test_every_wavefront_of_a_step_sees_the_same_count(sizes):
    """Steps right behind one another on tensors whose wavefronts end at different times: as with a wait after each of them."""
    made = _make(sizes, "bf16", "f32", 8, 16, fresh=True)
    desc, ends = adamw.make_desc(state_bits=8, seed=6), []
    for wait in (False, True):
        parts = _device(made)
        plan, step = _planned(desc, parts), torch.tensor([0], device="cuda")
        for _ in range(100):
            adamw.adamw_step(plan, step, 1e-3)
            if wait:
                torch.cuda.synchronize()
        assert int(step) == 100
        ends.append(_cpu(parts))
    for x, y in zip(*ends):
        for name in ("p", "m", "v", "m_exp", "v_exp"):
            assert torch.equal(x[name], y[name]), name


@gpu
def test_gradients_shared_by_two_tensors():
    made = _make([500, 500], "f32", "f32", 32, 13)
    parts = _device(made)
    parts[1]["g"] = parts[0]["g"]
    desc = adamw.make_desc()
    plan = _planned(desc, parts)
    before = _cpu(parts)
    adamw.adamw_step(plan, torch.tensor([1], device="cuda"), 1e-2)
    _check_step(before, _cpu(parts), desc, 2, 1e-2, 1.0)


@gpu
def test_elements_beyond_2_to_32():
    """One tensor whose last elements have numbers above 2^32, and a second one behind it."""
    n = (1 << 32) + 1000
    desc = adamw.make_desc(state_bits=8, seed=5)
    part = dict(p=torch.zeros(n, dtype=torch.bfloat16, device="cuda"), g=torch.ones(n, dtype=torch.bfloat16, device="cuda"))
    for k in ("m", "v"):
        part[k], part[k + "_exp"] = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(-(-n // 256), dtype=torch.uint8, device="cuda")
    made = _make([777], "bf16", "bf16", 8, 14)
    small = _device(made)[0]
    plan, norm = _planned(desc, [part, small]), torch.zeros(1, device="cuda")
    adamw.adamw_norm(plan, norm)
    want = math.sqrt(n + float(made[0]["g"].double().square().sum()))
    assert abs(float(norm) - want) <= 2 * U * want
    adamw.adamw_step(plan, torch.tensor([0], device="cuda"), 1e-2)
    # m' = 0.1, v' = 0.001, update 1e-2
    p1, m1, v1 = oracle.adamw_update(torch.zeros(1), torch.ones(1), torch.zeros(1), torch.zeros(1), 1, 1e-2, 0.9, 0.999, 1e-8, 0.0)
    for lo in (0, 1 << 31, (1 << 32) - 512, 1 << 32):
        cut = slice(lo, min(lo + 512, n))
        n_m, n_v, n_p = oracle.noise(5, 1, lo, cut.stop - lo)
        for name, x, got, digits, noise16 in (("p", p1, part["p"][cut].cpu(), 7, n_p),
                                              ("m", m1, oracle.held_value(part["m"][cut].cpu(), part["m_exp"][lo // 256: -(-cut.stop // 256)].cpu(), False), 3, n_m),
                                              ("v", v1, oracle.held_value(part["v"][cut].cpu(), part["v_exp"][lo // 256: -(-cut.stop // 256)].cpu(), True), 3, n_v)):
            x = x.expand(cut.stop - lo)
            _between(got, oracle.round_randomly(x * (1 - 32 * U), digits, noise16), oracle.round_randomly(x * (1 + 32 * U), digits, noise16), (name, lo))


# ---- lists that fill the card: four blocks a wavefront -------------------------------------------------------------------------------

# 8192 blocks are the most that a wavefront takes one at a time; the last ones end inside a wavefront's four blocks, inside a workgroup's sixteen and inside a block
FULL = [2047 * 1024 + 1, 1, 256, 255, 1023, 1025, 0, 4096, 4097, 16 * 256 * 3 - 1, 70001]


def test_lists_take_four_blocks_a_wavefront_from_8193_blocks_on():
    """What the tests below rely on, in the plan's size: a number for each piece of work of 4 x 1 or 4 x 4 blocks."""
    def size(blocks):
        b = ctypes.c_size_t()
        assert adamw.lib().adamw_query_bytes(ctypes.byref(adamw.make_desc()), _c_tensors(_part(n=256 * blocks)), 1, ctypes.byref(b)) == 0
        return b.value

    numbers = lambda pieces: -(-4 * pieces // 256) * 256  # noqa: E731
    rest = size(4) - numbers(1)
    assert size(8192) == rest + numbers(8192 // 4) and size(8193) == rest + numbers(-(-8193 // 16))
    assert sum(-(-n // 256) for n in FULL) > 8192


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p,g", KINDS)
def test_steps_of_lists_that_fill_the_card(p, g, bits):
    """As test_steps: a clipped step and one that is not, states of all kinds, nothing written behind a tensor's end."""
    desc = adamw.make_desc(0.9, 0.999, 1e-8, bits, seed=0xFEDCBA987654321)
    parts = _device(_make(FULL, p, g, bits, 21))
    guard = []
    for part in parts:
        for k in ("p", "master", "m", "v", "m_exp", "v_exp"):
            if k in part:
                t = part[k]
                wide = torch.empty(t.numel() + 64, dtype=t.dtype, device="cuda")
                wide.view(torch.uint8).fill_(0xA5)
                wide[: t.numel()] = t
                part[k] = wide[: t.numel()]
                guard.append((wide, t.numel()))
    plan, step, norm = _planned(desc, parts), torch.tensor([40], device="cuda"), torch.zeros(1, device="cuda")
    assert plan.c_plan.each == 4
    for n in range(2):
        before = _cpu(parts)
        adamw.adamw_norm(plan, norm)
        most = (float(norm) / 3, 0.0)[n]
        adamw.adamw_step(plan, step, 1e-2, norm=norm, max_norm=most)
        torch.cuda.synchronize()
        want = math.sqrt(sum(float(b["g"].double().square().sum()) for b in before))
        assert abs(float(norm) - want) <= 2 * U * want
        _check_step(before, _cpu(parts), desc, 41 + n, 1e-2, most / want if n == 0 else 1.0)
        assert int(step) == 41 + n
    for wide, n in guard:
        assert bool((wide[n:].view(torch.uint8) == 0xA5).all())


@gpu
def test_unpacked_states_of_a_list_that_fills_the_card():
    """Two blocks a wavefront at once, each with an exponent of its own; blocks of NaN among them."""
    made = _make(FULL, "bf16", "f32", 8, 22)
    for i, at in ((0, 0), (0, 5), (0, 8187), (9, 2)):
        made[i]["m_exp"][at] = 255
        made[i]["v_exp"][at + 1] = 255
    parts = _device(made)
    plan = _planned(adamw.make_desc(state_bits=8), parts)
    assert plan.c_plan.each == 4
    m, v = (torch.full((plan.elements,), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    adamw.adamw_unpack(plan, m, v)
    at = 0
    for part in made:
        n = part["p"].numel()
        for out, k, second in ((m, "m", False), (v, "v", True)):
            want = oracle.held_value(part[k], part[k + "_exp"], second)
            assert torch.equal(out[at: at + n].double().cpu().nan_to_num(nan=123.0), want.nan_to_num(nan=123.0))
            assert bool((out[at + n: at + -(-n // 256) * 256] == 0).all())
        at += -(-n // 256) * 256
    assert at == plan.elements


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_the_form_of_a_step_does_not_show_in_its_results(bits):
    """A tensor's step is the same bits in a short list and in one that fills the card, its elements having the same numbers."""
    made = _make([5000, 777, 2048, 1023], "bf16", "bf16", bits, 23)
    rest = _make([8192 * 256], "bf16", "bf16", bits, 24)
    desc, ends = adamw.make_desc(state_bits=bits, seed=31), []
    for more in ([], rest):
        parts = _device(made + more)
        plan = _planned(desc, parts)
        assert plan.c_plan.each == (4 if more else 1)
        adamw.adamw_step(plan, torch.tensor([12], device="cuda"), 1e-2)
        ends.append(_cpu(parts[: len(made)]))
    for x, y in zip(*ends):
        for k in set(x) - {"g", "weight_decay"}:
            assert torch.equal(x[k], y[k]), k
