"""LayerNorm of rows (lnorm.h) against its definition in 64 bits, and what its entry points refuse.

Tolerances.  u = 2^-24 is half a step of fp32, h half a step of the output's type relative to the value.  A sum in which no addend passes
through more than n additions is off by at most n u sum|addend|.  A row's values pass through at most 32 additions in a lane and 12 across
the lanes and wavefronts, and a few roundings: N = 64 covers a row's sums and what is computed from them.
With E = N u:  |err xh| <= E (mean|u| rstd + |xh|) =: e;  |err y| <= |gamma| e + 4 u (|gamma xh| + |beta|) + h |y|;
|err dx| <= rstd (E (|g| + mean|g|) + e |mean(g xh)| + |xh| (E mean|g xh| + mean(|g| e))) + E |dx| + h |dx| (dx with dsum).
Parameter gradients: a column's rows pass through at most rows / 8 additions before the partial sums and 256 behind them:
|err dgamma| <= (rows / 8 + 256) u sum|dy xh| + sum(|dy| e), |err dbeta| <= the first term of dy.
"""
import os

import pytest
import torch

from oracle import operators_oracle as oracle
from paper_2409_06206_amd import gswa, lnorm
from tests.test_abi_cpu import declared_functions

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
gpu = pytest.mark.gpu


# ---- without a GPU ---------------------------------------------------------------------------------------------------------------

def test_exports():
    assert set(declared_functions("lnorm.h", "lnorm")) == set(lnorm.EXPORTS)
    for n in lnorm.EXPORTS:
        assert hasattr(lnorm.lib(), n)


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), gswa.GSWA_EINVAL), (dict(rows=-1), gswa.GSWA_EINVAL), (dict(C=0), gswa.GSWA_EINVAL), (dict(dtype=2), gswa.GSWA_EINVAL),
    (dict(eps=-1.0), gswa.GSWA_EINVAL), (dict(eps=float("nan")), gswa.GSWA_EINVAL), (dict(flags=2), gswa.GSWA_EINVAL),
    (dict(x_stride=59), gswa.GSWA_EINVAL), (dict(y_stride=-60), gswa.GSWA_EINVAL), (dict(r_stride=1), gswa.GSWA_EINVAL),
    (dict(C=16385), gswa.GSWA_EUNSUPPORTED), (dict(C=16385, dtype="f32"), gswa.GSWA_EUNSUPPORTED),
    (dict(rows=1 << 40, C=60), gswa.GSWA_EUNSUPPORTED),
])
def test_bad_descriptors(change, status):
    with pytest.raises(gswa.GswaError) as e:
        lnorm.lnorm_query_bytes(lnorm.make_desc(**{**dict(rows=4, C=60, dtype="bf16"), **change}))
    assert e.value.status == status


@pytest.mark.parametrize("change", [dict(rows=1 << 64), dict(C=(1 << 32) + 60), dict(x_stride=(1 << 64) + 60), dict(flags=1 << 32), dict(dtype=1 << 32)])
def test_numbers_that_a_field_cannot_hold_are_refused(change):
    """Cut off to 32 or 64 bits they would be other, valid ones."""
    with pytest.raises(ValueError, match="hold"):
        lnorm.make_desc(**{**dict(rows=4, C=60, dtype="bf16"), **change})


def test_scratch_is_a_multiple_of_256():
    for rows, C in ((1, 1), (7, 60), (131072, 180), (4096, 16384)):
        n = lnorm.lnorm_query_bytes(lnorm.make_desc(rows, C, "bf16"))
        assert n > 0 and n % 256 == 0


def _addresses(n, gap=1 << 20, first=1 << 30):
    return [first + i * gap for i in range(n)]   # never dereferenced: the call is refused first


def test_bad_buffers_are_refused_before_a_launch():
    d = lnorm.make_desc(16, 60, "bf16")
    x, res, ga, be, y, s, dy, ds, dx, dg, db, ws = _addresses(12)

    def refused(call, *args):
        with pytest.raises(gswa.GswaError) as e:
            call(d, *args, stream=0)
        assert e.value.status == gswa.GSWA_EINVAL

    fwd, bwd = lnorm.lnorm_forward, lnorm.lnorm_backward
    refused(fwd, None, None, ga, be, y, None)
    refused(fwd, x, None, ga, be, None, None)
    refused(fwd, x, res, ga, be, y, None)              # a residual without a place for the sum
    refused(fwd, x, None, ga, be, y, s)
    refused(fwd, x + 2, None, ga, be, y, None)
    refused(fwd, x, None, ga, be, x, None)             # y over x
    refused(fwd, x, None, ga, be, ga - 16, None)
    refused(fwd, x, res, ga, be, y, y)
    refused(fwd, x, res, ga, be, y, x + 16)            # the sum may be x, not overlap it
    refused(fwd, x, res, ga, be, res, s)
    refused(bwd, x, dy, ga, ds, dx, dg, None, ws)
    refused(bwd, x, dy, ga, ds, dx, dg, db, None)
    refused(bwd, x, dy, ga, ds, dx, dg, db, ws + 16)
    refused(bwd, x, dy, ga, ds, x, dg, db, ws)
    refused(bwd, x, dy, ga, ds, dy + 16, dg, db, ws)
    refused(bwd, x, dy, ga, ds, dx, dg, dg + 16, ws)
    refused(bwd, x, dy, ga, ds, dx, dg, db, dg - 256)
    refused(bwd, x, dy, ga, ds, ws + 256, dg, db, ws)


def test_tensors_are_checked_against_the_descriptor():
    d = lnorm.make_desc(4, 8, "bf16")
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        lnorm.lnorm_forward(d, x, None, None, None, x.clone(), None, stream=0)


def test_what_a_descriptor_needs_follows_its_fields():
    """Found once for a descriptor's values, not for the object: a changed one is another."""
    d, other = lnorm.make_desc(4, 8, "bf16"), lnorm.make_desc(4, 8, "bf16")
    first = lnorm._specs.of(d)
    assert lnorm._specs.of(other) == first
    d.rows, d.y_stride = 5, 16
    spec = lnorm._specs.of(d)
    assert spec[2][0] == (5, 8) and spec[3] == ((5, 8), (16, 1)) and spec[5] == lnorm.lnorm_query_bytes(d)
    d.rows = 4
    d.y_stride = 0
    assert lnorm._specs.of(d) == first
    for rows in range(1, 1500):   # not more of them than a program has in use
        lnorm._specs.of(lnorm.make_desc(rows, 8, "f32"))
    assert len(lnorm._specs) <= lnorm._specs.MOST


# ---- on the GPU --------------------------------------------------------------------------------------------------------------------

def _strided(t, stride):
    """The same values in rows `stride` apart (0: close), NaN between them."""
    if not stride:
        return t.cuda()
    wide = torch.full((t.shape[0], stride), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, : t.shape[1]] = t.cuda()
    return wide[:, : t.shape[1]]


def _empty(rows, C, dtype, stride=0):
    return _strided(torch.full((rows, C), float("nan"), dtype=TYPE[dtype]), stride)


def _within(got, want, tol, what):
    got = got.detach().double().cpu()
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() / tol
    assert (over <= 1).all(), f"{what}: {float(over.max()):.3g} of the tolerance"


def _inputs(rows, C, dtype, seed, offset=0.0):
    gen = torch.Generator().manual_seed(seed)
    t = TYPE[dtype]
    new = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    scale = torch.exp(new(rows, 1))
    return dict(x=(new(rows, C) * scale + offset).to(t), residual=(new(rows, C) * scale).to(t), gamma=(1 + 0.3 * new(C)).to(t),
                beta=(0.3 * new(C)).to(t), dy=new(rows, C).to(t), dsum=new(rows, C).to(t))


def _check(rows, C, dtype, residual=False, affine=True, xs=0, ys=0, rs=0, eps=1e-5, seed=0, offset=0.0, wgrad=True):
    i = _inputs(rows, C, dtype, seed, offset)
    gamma, beta = (i["gamma"], i["beta"]) if affine else (None, None)
    dev = {k: _strided(i[k], {"x": xs, "dy": ys}.get(k, rs)) if i[k].dim() == 2 else i[k].cuda() for k in i}
    d = lnorm.make_desc(rows, C, dtype, eps, 0, xs, ys, rs)
    y, s, dx = _empty(rows, C, dtype, ys), _empty(rows, C, dtype, rs) if residual else None, _empty(rows, C, dtype, rs)
    lnorm.lnorm_forward(d, dev["x"], dev["residual"] if residual else None, dev["gamma"] if affine else None,
                        dev["beta"] if affine else None, y, s)
    u = i["x"]
    if residual:
        u = (i["x"].float() + i["residual"].float()).to(TYPE[dtype])
        assert torch.equal(s.cpu(), u)
    bd = lnorm.make_desc(rows, C, dtype, eps, 0, rs if residual else xs, ys, rs)
    dg, db = (torch.full((C,), float("nan"), device="cuda") for _ in range(2)) if wgrad else (None, None)
    ws = torch.full((lnorm.lnorm_query_bytes(bd),), 0x7F, dtype=torch.uint8, device="cuda")
    lnorm.lnorm_backward(bd, s if residual else dev["x"], dev["dy"], dev["gamma"] if affine else None, dev["dsum"] if residual else None,
                         dx, dg, db, ws if wgrad else None)
    torch.cuda.synchronize()
    want, xh, rstd = oracle.lnorm_forward(u, gamma, beta, eps)
    dxw, dgw, dbw = oracle.lnorm_backward(u, i["dy"], gamma, i["dsum"] if residual else None, eps)
    E, h = 64 * U, HALF[dtype]
    e = E * (u.double().abs().mean(1, keepdim=True) * rstd + xh.abs())
    ga, be = (gamma.double().abs(), beta.double().abs()) if affine else (torch.ones(C), torch.zeros(C))
    tiny = 1e-37
    _within(y, want, ga * e + 4 * U * (ga * xh.abs() + be) + h * want.abs() + tiny, "y")
    g = i["dy"].double() * (gamma.double() if affine else 1)
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    tol = rstd * (E * (g.abs() + mean(g.abs())) + e * mean(g * xh).abs() + xh.abs() * (E * mean((g * xh).abs()) + mean(g.abs() * e)))
    _within(dx, dxw, tol + (E + h) * dxw.abs() + tiny, "dx")
    if wgrad:
        n = (rows / 8 + 256) * U
        dy = i["dy"].double()
        _within(dg, dgw, n * (dy * xh).abs().sum(0) + (dy.abs() * e).sum(0) + tiny, "dgamma")
        _within(db, dbw, n * dy.abs().sum(0) + tiny, "dbeta")
    for t, ld in ((y, ys), (dx, rs), (s, rs)):   # nothing between the rows was written
        if t is not None and ld and rows > 1:
            between = torch.as_strided(t, (rows - 1, ld - C), (ld, 1), t.storage_offset() + C)
            assert torch.isnan(between).all()


# every width of the row variants and next to their borders; odd ones; C below a vector
WIDTHS = [1, 2, 3, 7, 8, 9, 31, 60, 64, 65, 127, 128, 129, 180, 192, 255, 256, 257, 360, 511, 512, 513, 1000, 1024, 1025, 1536, 2047, 2048, 2049, 4096,
          4100, 8191, 8192, 8193, 12289, 16383, 16384]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", WIDTHS)
def test_widths(C, dtype):
    _check(37 if C < 4096 else 5, C, dtype, residual=C % 2 == 0, seed=C)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 3, 16, 33, 1000, 4099])
@pytest.mark.parametrize("C", [60, 180, 333, 1030])
def test_numbers_of_rows(rows, C, dtype):
    _check(rows, C, dtype, residual=rows % 2 == 1, seed=rows)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("strides", [(70, 0, 0), (0, 61, 0), (0, 0, 67), (64, 73, 61)])
@pytest.mark.parametrize("residual", [False, True])
def test_strides(strides, dtype, residual):
    _check(29, 60, dtype, residual, xs=strides[0], ys=strides[1], rs=strides[2], seed=3)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_gamma_and_beta_and_without_their_gradients(dtype):
    _check(17, 100, dtype, affine=False, seed=5)
    _check(17, 100, dtype, residual=True, wgrad=False, seed=6)


@gpu
def test_a_mean_far_from_zero():
    """Squares are of distances from the mean: a mean of 1000 deviations leaves the variance its digits."""
    _check(64, 768, "f32", offset=1000.0, seed=7)


@gpu
def test_rows_of_equal_values_and_of_extreme_ones():
    C = 60
    x = torch.stack([torch.full((C,), 3.0), torch.zeros(C), torch.full((C,), -3e36), torch.linspace(-1e37, 1e37, C), torch.linspace(0, 1e-40, C),
                     torch.ones(C), torch.ones(C)])
    x[5, 3], x[6, 9] = float("nan"), float("inf")
    d, y = lnorm.make_desc(7, C, "f32"), torch.empty(7, C, device="cuda")
    beta = torch.linspace(-1, 1, C)
    lnorm.lnorm_forward(d, x.cuda(), None, None, beta.cuda(), y, None)
    y = y.cpu()
    assert torch.equal(y[:3], beta.expand(3, C))            # nothing but beta where all distances are 0
    assert torch.equal(y[3], beta)                          # or where their squares overflow
    assert (y[4] - beta).abs().max() < 1e-30                # eps is what divides
    assert torch.isnan(y[5]).all() and torch.isnan(y[6]).all()   # of their row, as the formula has it
    assert not torch.isnan(y[:5]).any()


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [60, 180, 333, 1281, 1539, 4099, 12289])   # last vectors that begin in another wavefront's among them
def test_in_place(C, dtype):
    rows = 700 if C < 4096 else 300
    i = {k: v.cuda() for k, v in _inputs(rows, C, dtype, 1).items()}
    d = lnorm.make_desc(rows, C, dtype)
    new = lambda: torch.empty_like(i["x"])  # noqa: E731
    y, s, dx, y2 = new(), new(), new(), new()
    lnorm.lnorm_forward(d, i["x"], i["residual"], i["gamma"], i["beta"], y, s)
    for over in ("x", "residual"):
        j = {k: v.clone() for k, v in i.items()}
        lnorm.lnorm_forward(d, j["x"], j["residual"], j["gamma"], j["beta"], y2, j[over])
        assert torch.equal(y, y2) and torch.equal(s, j[over])
    dg, db, dg2, db2 = (torch.empty(C, device="cuda") for _ in range(4))
    ws = torch.empty(lnorm.lnorm_query_bytes(d), dtype=torch.uint8, device="cuda")
    lnorm.lnorm_backward(d, s, i["dy"], i["gamma"], i["dsum"], dx, dg, db, ws)
    for over in ("dy", "dsum"):
        j = {k: v.clone() for k, v in i.items()}
        lnorm.lnorm_backward(d, s, j["dy"], j["gamma"], j["dsum"], j[over], dg2, db2, ws)
        assert torch.equal(dx, j[over]) and torch.equal(dg, dg2) and torch.equal(db, db2)


@gpu
def test_accumulated_gradients_and_the_same_bits_every_run():
    i = {k: v.cuda() for k, v in _inputs(3001, 333, "bf16", 2).items()}
    d, da = lnorm.make_desc(3001, 333, "bf16"), lnorm.make_desc(3001, 333, "bf16", flags=lnorm.LNORM_ACCUM_WGRAD)
    ws = torch.empty(lnorm.lnorm_query_bytes(d), dtype=torch.uint8, device="cuda")
    dx, dg, db = torch.empty_like(i["x"]), torch.empty(333, device="cuda"), torch.empty(333, device="cuda")
    lnorm.lnorm_backward(d, i["x"], i["dy"], i["gamma"], None, dx, dg, db, ws)
    for _ in range(3):
        g2, b2 = torch.ones(333, device="cuda"), torch.zeros(333, device="cuda")
        lnorm.lnorm_backward(da, i["x"], i["dy"], i["gamma"], None, dx, g2, b2, ws)
        assert torch.equal(g2, 1 + dg) and torch.equal(b2, db)


@gpu
def test_gradients_by_differences():
    """Central differences of sum(w y) of the definition in 64 bits, in random directions of x, gamma and beta, against the kernels'
    fp32 gradients."""
    gen = torch.Generator().manual_seed(4)
    rows, C, eps = 6, 40, 1e-5
    x, gamma, beta, w = (torch.randn(*s, generator=gen) for s in ((rows, C), (C,), (C,), (rows, C)))
    d = lnorm.make_desc(rows, C, "f32", eps)
    ws = torch.empty(lnorm.lnorm_query_bytes(d), dtype=torch.uint8, device="cuda")
    dx, dg, db = torch.empty(rows, C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    lnorm.lnorm_backward(d, x.cuda(), w.cuda(), gamma.cuda(), None, dx, dg, db, ws)
    loss = lambda x, ga, be: float((oracle.lnorm_forward(x, ga, be, eps)[0] * w.double()).sum())  # noqa: E731
    step = 1e-5   # truncation ~ step^2, rounding ~ 2^-53 / step: both far below the fp32 gradients' own 64 u
    for k, got in enumerate((dx, dg, db)):
        args = [x.double(), gamma.double(), beta.double()]
        v = torch.randn(args[k].shape, generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + step * v, args[k] - step * v
        want = (loss(*up) - loss(*down)) / (2 * step)
        have = got.double().cpu()
        scale = float((have.abs() * v.abs()).sum())
        assert abs(float((have * v).sum()) - want) <= 64 * U * 4 * scale + 1e-8 * abs(want)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 7, 60, 131, 180, 391, 768, 1531, 2048, 2999, 4100, 8192])
def test_gradients_of_one_workgroup_and_of_several_are_added_up(C, dtype):
    """From one row, that one workgroup has, to enough for several: what is added is the plain call's, rounded once more."""
    for rows in (1, 2, 5, 16, 70, 300):
        i = {k: v.cuda() for k, v in _inputs(rows, C, dtype, 30).items()}
        ws = torch.empty(lnorm.lnorm_query_bytes(lnorm.make_desc(rows, C, dtype)), dtype=torch.uint8, device="cuda")
        first = [torch.randn(C, device="cuda") for _ in range(2)]
        plain, added, dx = [torch.full((C,), float("nan"), device="cuda") for _ in range(2)], [t.clone() for t in first], torch.empty_like(i["x"])
        lnorm.lnorm_backward(lnorm.make_desc(rows, C, dtype), i["x"], i["dy"], i["gamma"], None, dx, *plain, ws)
        lnorm.lnorm_backward(lnorm.make_desc(rows, C, dtype, flags=lnorm.LNORM_ACCUM_WGRAD), i["x"], i["dy"], i["gamma"], None, dx, *added, ws)
        for p, f, t in zip(plain, first, added):
            assert torch.equal(t, f + p), (rows, C)


@gpu
def test_other_streams_and_a_replayed_graph():
    """Two streams at once with buffers of their own; a captured pass replayed on new values between eager calls."""
    cases = []
    for seed, (rows, C) in enumerate(((513, 180), (64, 2048))):
        i = {k: v.cuda() for k, v in _inputs(rows, C, "bf16", 20 + seed).items()}
        d = lnorm.make_desc(rows, C, "bf16")
        buf = lambda: dict(y=torch.zeros_like(i["x"]), sum=torch.zeros_like(i["x"]), dx=torch.zeros_like(i["x"]),  # noqa: E731
                           dg=torch.zeros(C, device="cuda"), db=torch.zeros(C, device="cuda"),
                           ws=torch.zeros(lnorm.lnorm_query_bytes(d), dtype=torch.uint8, device="cuda"))
        cases.append((d, i, buf(), buf()))

    def run(d, i, o, stream=None):
        lnorm.lnorm_forward(d, i["x"], i["residual"], i["gamma"], i["beta"], o["y"], o["sum"], stream)
        lnorm.lnorm_backward(d, o["sum"], i["dy"], i["gamma"], i["dsum"], o["dx"], o["dg"], o["db"], o["ws"], stream)

    same = lambda a, b: all(torch.equal(a[k], b[k]) for k in a if k != "ws")  # noqa: E731
    for d, i, want, _ in cases:
        run(d, i, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        for s, (d, i, _, got) in zip(streams, cases):
            run(d, i, got, s)
    torch.cuda.synchronize()
    assert all(same(w, g) for _, _, w, g in cases)
    d, i, want, got = cases[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(d, i, got)
    for k in range(4):
        i["x"].copy_(torch.randn(i["x"].shape, generator=torch.Generator().manual_seed(k)))
        for t in got.values():
            t.zero_()
        graph.replay()
        run(d, i, want)
        torch.cuda.synchronize()
        assert same(want, got), k


@gpu
def test_more_than_2_to_31_elements():
    rows, C = 1_100_000, 2048
    x = torch.empty(rows, C, dtype=torch.bfloat16, device="cuda").normal_()
    y = torch.empty_like(x)
    d = lnorm.make_desc(rows, C, "bf16")
    lnorm.lnorm_forward(d, x, None, None, None, y, None)
    at = torch.tensor([0, 1, 524288, 1_048_575, 1_048_576, 1_048_577, rows - 1], device="cuda")
    want, _, _ = oracle.lnorm_forward(x[at].cpu(), None, None, 1e-5)
    assert ((y[at].double().cpu() - want).abs() <= HALF["bf16"] * want.abs() + 1e-5).all()
    dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = torch.empty(lnorm.lnorm_query_bytes(d), dtype=torch.uint8, device="cuda")
    dy = torch.ones(1, C, dtype=torch.bfloat16, device="cuda").expand(rows, C).contiguous()
    lnorm.lnorm_backward(d, x, dy, None, None, y, dg, db, ws)
    assert torch.equal(db, torch.full((C,), float(rows), device="cuda"))   # whole numbers below 2^24: exact in any order
    # dy the same in all of a row: g - mean g = 0 and mean(g xh) = mean xh = 0 up to E
    assert float(y.abs().max()) < 64 * U * 16


# ---- more rows than the workgroups take at once -----------------------------------------------------------------------------------

# Workgroups of the forward pass: at most 1024 for rows on 512 lanes, 2048 for others, of 1 to 32 rows each; of the backward pass 256 to 768.
ROUNDS = {"bf16": [(1100, 12289), (1031, 6150), (2100, 5001), (2053, 3080), (4200, 1539), (8300, 780), (17000, 333), (70001, 60)],
          "f32": [(1100, 12289), (1031, 4100), (2100, 2501), (4200, 1531), (8300, 780), (17000, 333), (70001, 60)]}
ROUNDS = [(dtype, rows, C) for dtype, shapes in ROUNDS.items() for rows, C in shapes]


@gpu
@pytest.mark.parametrize("dtype,rows,C", ROUNDS)
@pytest.mark.parametrize("residual", [False, True])
def test_workgroups_that_go_on_to_further_rows(dtype, rows, C, residual):
    _check(rows, C, dtype, residual, seed=C)


@gpu
@pytest.mark.parametrize("dtype,rows,C", ROUNDS)
def test_in_place_over_further_rows(dtype, rows, C):
    """The next row is read while this one's sum is stored: over x or the residual, and dx over dy or dsum, as into buffers of their own."""
    i = {k: v.cuda() for k, v in _inputs(rows, C, dtype, 41).items()}
    d = lnorm.make_desc(rows, C, dtype)
    y, s, dx, y2 = (torch.empty_like(i["x"]) for _ in range(4))
    lnorm.lnorm_forward(d, i["x"], i["residual"], i["gamma"], i["beta"], y, s)
    assert torch.equal(s, (i["x"].float() + i["residual"].float()).to(TYPE[dtype]))
    for over in ("x", "residual"):
        j = {k: i[k].clone() for k in ("x", "residual")}
        lnorm.lnorm_forward(d, j["x"], j["residual"], i["gamma"], i["beta"], y2, j[over])
        assert torch.equal(y, y2) and torch.equal(s, j[over]), over
    dg, db, dg2, db2 = (torch.empty(C, device="cuda") for _ in range(4))
    ws = torch.empty(lnorm.lnorm_query_bytes(d), dtype=torch.uint8, device="cuda")
    lnorm.lnorm_backward(d, s, i["dy"], i["gamma"], i["dsum"], dx, dg, db, ws)
    for over in ("dy", "dsum"):
        j = {k: i[k].clone() for k in ("dy", "dsum")}
        lnorm.lnorm_backward(d, s, j["dy"], i["gamma"], j["dsum"], j[over], dg2, db2, ws)
        assert torch.equal(dx, j[over]) and torch.equal(dg, dg2) and torch.equal(db, db2), over
