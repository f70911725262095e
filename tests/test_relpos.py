"""Relative position bias by buckets (relpos.h) against its definition, and what its entry points refuse.

The forward pass copies values: equal to the bit.  Gradients are taken of whole numbers of at most 7 bits and random sign, whose sums stay far
below 2^24: exact in fp32 in any order, so they are equal too; one test takes normal numbers, with a tolerance.
"""
import math

import pytest
import torch

from oracle import operators_oracle as oracle
from paper_2409_06206_amd import gswa, relpos
from tests.test_abi_cpu import declared_functions

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BI, CAUSAL, ACCUM = relpos.RELPOS_BIDIRECTIONAL, relpos.RELPOS_CAUSAL, relpos.RELPOS_ACCUM_WGRAD
gpu = pytest.mark.gpu


# ---- without a GPU ---------------------------------------------------------------------------------------------------------------

def test_exports():
    assert set(declared_functions("relpos.h", "relpos")) == set(relpos.EXPORTS)
    for n in relpos.EXPORTS:
        assert hasattr(relpos.lib(), n)


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("distance", [3, 7, 16, 64, 65, 100, 127, 128, 129, 512, 800, 4096, 46341, 1 << 20, (1 << 31) - 1])
def test_log_edges_are_found_in_whole_numbers(distance, both):
    """Powers of two and of ten put borders exactly on whole numbers, where a rounded logarithm would decide by chance."""
    for buckets in (2, 3, 4, 5, 8, 10, 16, 32, 63, 64, 128, 256):
        side = buckets // 2 if both else buckets
        if (both and buckets % 2) or not 2 <= side <= 128 or distance <= side // 2:
            with pytest.raises(gswa.GswaError):
                relpos.relpos_log_edges(buckets, distance, both)
            continue
        edges = relpos.relpos_log_edges(buckets, distance, both)
        assert edges == oracle.log_edge(buckets, distance, both)
        assert len(edges) == side - 1


def test_log_edges_of_the_usual_sizes():
    assert relpos.relpos_log_edges(32, 128, True) == [1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 23, 32, 46, 64, 91]
    assert relpos.relpos_log_edges(8, 64, False) == [1, 2, 3, 4, 8, 16, 32]


GOOD = dict(heads=4, edges=[1, 2, 4], dtype="bf16", flags=BI, q_len=5, k_len=7)


@pytest.mark.parametrize("change,status", [
    (dict(heads=0), -1), (dict(heads=65536), -1), (dict(dtype=3), -1), (dict(flags=8), -1), (dict(q_len=0), -1), (dict(k_len=-1), -1),
    (dict(q_start=-1), -1), (dict(batch=0), -1), (dict(row_stride=6), -1), (dict(edges=[0, 1]), -1), (dict(edges=[2, 1]), -1),
    (dict(window=-1), -1), (dict(window=65), -1), (dict(window=8, flags=0), -1), (dict(window=8, flags=BI | CAUSAL), -1),
    (dict(window=8, heads=4097), -2), (dict(q_len=1 << 30, q_start=1), -2), (dict(heads=60000, batch=60000, q_len=60000, k_len=60000), -2),
])
def test_bad_descriptors(change, status):
    with pytest.raises(gswa.GswaError) as e:
        relpos.relpos_query_bytes(relpos.make_desc(**{**GOOD, **change}))
    assert e.value.status == status


def test_too_many_edges():
    with pytest.raises(ValueError):
        relpos.make_desc(1, list(range(1, 129)), "f32", q_len=1, k_len=1)


@pytest.mark.parametrize("change", [dict(q_start=(1 << 32) + 5), dict(heads=(1 << 32) + 4), dict(edges=[1, (1 << 32) + 4]), dict(batch=1 << 32),
                                    dict(row_stride=(1 << 64) + 7), dict(window=-(1 << 32) + 8)])
def test_numbers_that_a_field_cannot_hold_are_refused(change):
    """Cut off to 32 or 64 bits they would be other, valid ones."""
    with pytest.raises(ValueError, match="hold"):
        relpos.make_desc(**{**GOOD, **change})
    for buckets, distance in ((32, (1 << 32) + 128), ((1 << 32) + 32, 128), (32, 1 << 31)):
        with pytest.raises(ValueError, match="hold"):
            relpos.relpos_log_edges(buckets, distance, True)


def test_bad_buffers_are_refused_before_a_launch():
    d = relpos.make_desc(**GOOD)
    size = relpos.relpos_query_bytes(d)
    assert size > 0 and size % 256 == 0
    table, out, dout, dt, ws = (1 << 30, 1 << 31, 3 << 30, 1 << 32, 5 << 30)

    def refused(call, *args):
        with pytest.raises(gswa.GswaError) as e:
            call(d, *args, stream=0)
        assert e.value.status == gswa.GSWA_EINVAL

    refused(relpos.relpos_forward, None, out)
    refused(relpos.relpos_forward, table, None)
    refused(relpos.relpos_forward, table, table + 16)
    refused(relpos.relpos_forward, table + 2, out)
    refused(relpos.relpos_backward, dout, None, ws)
    refused(relpos.relpos_backward, dout, dt, None)
    refused(relpos.relpos_backward, dout, dt, ws + 16)
    refused(relpos.relpos_backward, dout, dout + 16, ws)
    refused(relpos.relpos_backward, dout, ws, ws)
    refused(relpos.relpos_backward, ws, dt, ws)


# ---- on the GPU --------------------------------------------------------------------------------------------------------------------

def _whole(shape, dtype, seed):
    return torch.randint(-64, 65, shape, generator=torch.Generator().manual_seed(seed)).to(TYPE[dtype])


def _check(heads, q, k, start, edges, dtype, flags=0, batch=1, pad=0, seed=0):
    both, causal = bool(flags & BI), bool(flags & CAUSAL)
    ld = k + pad
    d = relpos.make_desc(heads, edges, dtype, flags, q, k, start, batch, row_stride=ld if pad else 0)
    table = torch.randn(d.buckets, heads, generator=torch.Generator().manual_seed(seed)).to(TYPE[dtype])
    out = torch.full((heads * q, ld), 77.0, dtype=TYPE[dtype], device="cuda")
    relpos.relpos_forward(d, table.cuda(), out[:, :k])
    want = oracle.sequence_forward(table, q, k, start, edges, both, causal)
    assert torch.equal(out[:, :k].cpu().view(heads, q, k), want)
    assert bool((out[:, k:] == 77).all())
    dout = _whole((batch, heads, q, k), dtype, seed + 1)
    wide = torch.full((batch * heads * q, ld), float("nan"), dtype=TYPE[dtype], device="cuda")
    wide[:, :k] = dout.view(-1, k).cuda()
    if causal:   # what stands where nothing is seen is not read
        hidden = torch.arange(k)[None, :] > torch.arange(q)[:, None] + start
        wide.view(batch, heads, q, ld)[..., :k][..., hidden.cuda()] = float("nan")
    got = torch.full((d.buckets, heads), float("nan"), device="cuda")
    ws = torch.full((relpos.relpos_query_bytes(d),), 0x7F, dtype=torch.uint8, device="cuda")
    relpos.relpos_backward(d, wide[:, :k], got, ws)
    dwant = oracle.sequence_backward(dout, start, edges, both, causal, d.buckets)
    assert torch.equal(got.double().cpu(), dwant)
    da = relpos.make_desc(heads, edges, dtype, flags | ACCUM, q, k, start, batch, row_stride=ld if pad else 0)
    relpos.relpos_backward(da, wide[:, :k], got, ws)
    assert torch.equal(got.double().cpu(), 2 * dwant)


LOG = {n: oracle.log_edge(*n) for n in ((32, 128, True), (32, 128, False), (64, 800, True), (256, 2048, True), (128, 300, False))}


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("flags", [0, BI, CAUSAL, BI | CAUSAL])
@pytest.mark.parametrize("q,k,start", [(1, 1, 0), (1, 1, 5), (1, 515, 514), (1, 515, 100), (7, 3, 0), (64, 64, 0), (65, 129, 0), (129, 1031, 902),
                                       (200, 77, 0), (300, 300, 1000), (333, 517, 3), (1024, 640, 0)])
def test_lengths(q, k, start, flags, dtype):
    _check(3, q, k, start, LOG[32, 128, bool(flags & BI)], dtype, flags, batch=2, seed=q + k)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", list(LOG))
def test_edges(n, dtype):
    _check(2, 411, 1203, 17, LOG[n], dtype, BI if n[2] else 0, seed=1)
    _check(2, 1203, 411, 0, LOG[n], dtype, BI if n[2] else CAUSAL, seed=2)


@gpu
@pytest.mark.parametrize("edges", [[], [1], [5], [1, 1, 1, 2], [3, 3, 900], list(range(1, 128)), [1 << 30]])
@pytest.mark.parametrize("flags", [0, BI, CAUSAL])
def test_any_ascending_edges(edges, flags):
    _check(2, 70, 1000, 400, edges, "bf16", flags, seed=len(edges))


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [1, 3, 8, 64])
def test_rows_apart(pad, dtype):
    _check(2, 90, 301, 0, LOG[32, 128, True], dtype, BI, batch=3, pad=pad)
    _check(2, 90, 296, 210, LOG[32, 128, False], dtype, CAUSAL, batch=2, pad=pad)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [31, 32, 33, 63, 64, 65, 66, 95, 127, 129, 200, 255, 257, 480, 511, 512, 513, 575, 1000, 1023, 1025, 1055, 1087, 1531, 2039, 2047, 2049,
                               2111, 4097])
def test_rows_right_behind_one_another_from_any_place(k, dtype):
    """Rows that start anywhere in a line and run into the next one: every element once, nothing before the first and behind the last."""
    edges = list(range(1, 120))   # (a bucket for each offset near the diagonal, which passes through all row ends here)
    size = torch.tensor([], dtype=TYPE[dtype]).element_size()
    for n, (heads, q) in enumerate(((3, 1), (1, 2), (2, 9), (2, 65), (1, 200))):
        for start in (0, k - 40 if k > 40 else 3):
            for place in ((0, 16, 48, 112) if q == 9 else (16 * (n + 1),)):   # bytes behind a line's start
                d = relpos.make_desc(heads, edges, dtype, BI, q, k, start)
                table = torch.randn(d.buckets, heads, generator=torch.Generator().manual_seed(k)).to(TYPE[dtype])
                room = torch.full((heads * q * k + 512,), 77.0, dtype=TYPE[dtype], device="cuda")
                first = 128 // size + place // size
                assert room.data_ptr() % 128 == 0
                relpos.relpos_forward(d, table.cuda(), room[first: first + heads * q * k])
                want = oracle.sequence_forward(table, q, k, start, edges, True, False)
                assert torch.equal(room[first: first + heads * q * k].cpu().view(heads, q, k), want), (heads, q, start, place)
                assert bool((room[:first] == 77).all()) and bool((room[first + heads * q * k:] == 77).all())


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q", [1, 2, 7, 8])
def test_few_rows_apart(q, dtype):
    for k, pad in ((5, 2), (515, 1), (515, 61), (1027, 5), (2100, 76)):
        _check(3, q, k, k - q if k > q else 0, LOG[32, 128, False], dtype, CAUSAL, batch=2, pad=pad)


@gpu
def test_heads_and_images():
    for heads, batch in ((1, 5), (17, 1), (64, 3)):
        _check(heads, 40, 300, 260, LOG[32, 128, True], "bf16", BI, batch=batch)


@gpu
def test_every_query_before_the_first_key_but_one():
    """A prefix that is not there: with q_start = 0 the first query sees key 0 alone."""
    _check(2, 5, 2000, 0, LOG[32, 128, False], "f32", CAUSAL)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,heads,buckets,distance", [(1, 1, 4, 3), (2, 3, 8, 5), (8, 6, 10, 6), (12, 4, 32, 128), (16, 6, 18, 14), (33, 16, 24, 20),
                                                       (64, 2, 256, 65), (64, 31, 6, 3)])
def test_windows(M, heads, buckets, distance, dtype):
    edges = oracle.log_edge(buckets, distance, True)
    d = relpos.make_desc(heads, edges, dtype, BI, window=M)
    at = oracle.window_bucket(M, edges)
    table = torch.randn(d.buckets, heads, generator=torch.Generator().manual_seed(M)).to(TYPE[dtype])
    out = torch.empty(at.numel(), heads, dtype=TYPE[dtype], device="cuda")
    relpos.relpos_forward(d, table.cuda(), out)
    assert torch.equal(out.cpu(), table[at])
    dout = _whole((at.numel(), heads), "f32", M)
    got = torch.full((d.buckets, heads), float("nan"), device="cuda")
    relpos.relpos_backward(d, dout.cuda(), got, None if relpos.relpos_query_bytes(d) == 0 else
                           torch.empty(relpos.relpos_query_bytes(d), dtype=torch.uint8, device="cuda"))
    want = torch.zeros(d.buckets, heads).index_add_(0, at, dout)
    assert torch.equal(got.cpu(), want)
    da = relpos.make_desc(heads, edges, dtype, BI | ACCUM, window=M)
    relpos.relpos_backward(da, dout.cuda(), got, None if relpos.relpos_query_bytes(d) == 0 else
                           torch.empty(relpos.relpos_query_bytes(d), dtype=torch.uint8, device="cuda"))
    assert torch.equal(got.cpu(), 2 * want)


@gpu
def test_window_tables_are_those_of_the_attention_layer():
    """With a bucket for every distance the table of buckets is gswa.h's own, in another order: row (key - query) of one axis sits at
    |d| or, behind the query, at M + d."""
    M, heads = 8, 6
    edges = list(range(1, M))
    d = relpos.make_desc(heads, edges, "f32", BI, window=M)
    table = torch.randn(d.buckets, heads, generator=torch.Generator().manual_seed(0))
    out = torch.empty((2 * M - 1) ** 2, heads, device="cuda")
    relpos.relpos_forward(d, table.cuda(), out)
    out = out.cpu()
    row = lambda r: -r if r <= 0 else M + r  # noqa: E731
    for n, m in (((0, 0), (7, 7)), ((3, 2), (3, 5)), ((7, 1), (0, 6)), ((4, 4), (4, 4))):   # (row, column) of a query and of a key
        idx = (n[0] - m[0] + M - 1) * (2 * M - 1) + (n[1] - m[1] + M - 1)
        assert torch.equal(out[idx], table[row(m[0] - n[0]) * 2 * M + row(m[1] - n[1])])


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_normal_numbers_and_the_same_bits_every_run(dtype):
    """A value passes through at most 64 additions down a diagonal or 4096 / 8 along a row, 256 in a workgroup, and sums in fp64 behind them:
    off by at most (512 + 256 + 16) 2^-24 of the sum of magnitudes."""
    q, k, edges = 700, 4096, LOG[32, 128, True]
    dout = torch.randn(2, 4, q, k, generator=torch.Generator().manual_seed(9)).to(TYPE[dtype])
    d = relpos.make_desc(4, edges, dtype, BI, q, k, 1500, 2)
    ws = torch.empty(relpos.relpos_query_bytes(d), dtype=torch.uint8, device="cuda")
    got, dev = [torch.empty(d.buckets, 4, device="cuda") for _ in range(3)], dout.cuda()
    for g in got:
        relpos.relpos_backward(d, dev, g, ws)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    want = oracle.sequence_backward(dout, 1500, edges, True, False, d.buckets)
    size = oracle.sequence_backward(dout.abs(), 1500, edges, True, False, d.buckets)
    assert ((got[0].double().cpu() - want).abs() <= 784 * 2.0 ** -24 * size).all()


@gpu
def test_infinities_and_nan_stay_in_their_bucket():
    edges = LOG[32, 128, True]
    d = relpos.make_desc(1, edges, "f32", BI, 300, 300)
    dout = torch.zeros(1, 1, 300, 300)
    dout[0, 0, 10, 290], dout[0, 0, 150, 147], dout[0, 0, 299, 0] = math.nan, math.inf, -math.inf
    got = torch.empty(d.buckets, 1, device="cuda")
    relpos.relpos_backward(d, dout.cuda(), got, torch.empty(relpos.relpos_query_bytes(d), dtype=torch.uint8, device="cuda"))
    got = got.cpu()[:, 0]
    at = oracle.bucket(torch.tensor([280, -3, -299]), edges, True)
    assert torch.isnan(got[at[0]]) and got[at[1]] == math.inf and got[at[2]] == -math.inf
    got[at] = 0
    assert bool((got == 0).all())


@gpu
def test_more_than_2_to_31_elements():
    heads, q, k, edges = 9, 16000, 16001, LOG[32, 128, True]
    d = relpos.make_desc(heads, edges, "bf16", BI, q, k, 3)
    table = torch.randn(d.buckets, heads, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    out = torch.empty(heads, q, k, dtype=torch.bfloat16, device="cuda")
    relpos.relpos_forward(d, table.cuda(), out)
    for i in (0, 1, 8000, 15999):
        b = oracle.bucket(torch.arange(k) - i - 3, edges, True)
        assert torch.equal(out[:, i].cpu(), table[b].t())
    out.fill_(0)
    out[8, 15999, 0], out[8, 15999, 16000], out[7, 3, 5], out[8, 15990, 15993] = 3, 5, 7, 11
    got = torch.empty(d.buckets, heads, device="cuda")
    relpos.relpos_backward(d, out, got, torch.empty(relpos.relpos_query_bytes(d), dtype=torch.uint8, device="cuda"))
    want = torch.zeros(d.buckets, heads)
    for h, i, j, v in ((8, 15999, 0, 3), (8, 15999, 16000, 5), (7, 3, 5, 7), (8, 15990, 15993, 11)):
        want[oracle.bucket(torch.tensor([j - i - 3]), edges, True)[0], h] += v
    assert torch.equal(got.cpu(), want)


@gpu
def test_other_streams_and_a_replayed_graph():
    edges = LOG[32, 128, True]
    ds = [relpos.make_desc(4, edges, "bf16", BI, 257, 300, 11, 2), relpos.make_desc(6, oracle.log_edge(18, 14, True), "bf16", BI, window=16)]
    cases = []
    for n, d in enumerate(ds):
        shape = (4, 257, 300) if n == 0 else (961, 6)
        table = torch.randn(d.buckets, d.heads, generator=torch.Generator().manual_seed(n)).to(torch.bfloat16).cuda()
        dout = _whole((2,) + shape if n == 0 else shape, "bf16" if n == 0 else "f32", n).cuda()
        new = lambda: (torch.zeros(shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(d.buckets, d.heads, device="cuda"),  # noqa: E731
                       torch.empty(relpos.relpos_query_bytes(d) + 256, dtype=torch.uint8, device="cuda"))
        cases.append((d, table, dout, new(), new()))

    def run(d, table, dout, o, stream=None):
        relpos.relpos_forward(d, table, o[0], stream)
        relpos.relpos_backward(d, dout, o[1], o[2], stream)

    for d, table, dout, want, _ in cases:
        run(d, table, dout, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for s, (d, table, dout, _, got) in zip(streams, cases):
            run(d, table, dout, got, s)
    torch.cuda.synchronize()
    for _, _, _, want, got in cases:
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    for d, table, dout, want, got in cases:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(d, table, dout, got)
        for k in range(4):
            table.copy_(torch.randn(table.shape, generator=torch.Generator().manual_seed(100 + k)))
            dout.copy_(_whole(dout.shape, "f32", 100 + k))
            got[0].zero_(), got[1].zero_()
            graph.replay()
            run(d, table, dout, want)
            torch.cuda.synchronize()
            assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]), k


# ---- workgroups of 256 threads, tiles of many rows ---------------------------------------------------------------------------------

def _check_forward(heads, q, k, start, edges, dtype, flags=0, pad=0, place=0, seed=0):
    """All of the bias, held against the definition on the GPU (too much for the CPU); `place`: bytes behind a line's start."""
    both, causal = bool(flags & BI), bool(flags & CAUSAL)
    ld, size = k + pad, torch.tensor([], dtype=TYPE[dtype]).element_size()
    d = relpos.make_desc(heads, edges, dtype, flags, q, k, start, row_stride=ld if pad else 0)
    table = torch.randn(d.buckets, heads, generator=torch.Generator().manual_seed(seed)).to(TYPE[dtype]).cuda()
    first, count = (128 + place) // size, heads * q * ld
    room = torch.full((count + 512,), 77.0, dtype=TYPE[dtype], device="cuda")
    assert room.data_ptr() % 128 == 0
    rows = room[first: first + count].view(heads * q, ld)
    relpos.relpos_forward(d, table, rows[:, :k] if pad else rows)
    at = oracle.sequence_bucket(q, k, start, edges, both).cuda()
    hidden = torch.arange(k, device="cuda")[None, :] > torch.arange(q, device="cuda")[:, None] + start
    for h in range(heads):
        want = table[:, h][at]
        if causal:
            want[hidden] = -math.inf
        assert torch.equal(rows.view(heads, q, ld)[h, :, :k], want), h
    assert bool((rows[:, k:] == 77).all())
    assert bool((room[:first] == 77).all()) and bool((room[first + count:] == 77).all())


# Workgroups have 256 threads where a row is longer than a wavefront's vectors (512 values in bf16, 256 in fp32) and 8 rows a tile make 512 of them or more.
WIDE = {"bf16": (520, 1000, 1023, 1024, 1025, 2048, 2049, 2113, 4100), "f32": (260, 515, 1000, 1023, 1024, 1025, 1056, 2049, 2113)}


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", range(9))
def test_workgroups_of_256_threads(n, dtype):
    """Rows from a line's start, right behind one another from any place, and with something between them."""
    k, near = WIDE[dtype][n], list(range(1, 120))
    for heads, q, pad, place, flags in ((9, 512, 0, 0, BI), (9, 515, 0, 16, CAUSAL), (10, 483, 0, 112, BI), (9, 512, -k % 64, 0, BI), (9, 517, 1, 0, BI),
                                        (9, 513, 3, 48, CAUSAL), (11, 480, 70, 16, 0)):
        _check_forward(heads, q, k, k - 300 if n % 2 else 0, near, dtype, flags, pad, place, seed=n)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 5, None])   # None: rows that start at lines
def test_tiles_of_64_rows(pad, dtype):
    """Enough workgroups for the largest tiles, the last of which is short; bands of rows spread over the XCDs with some left over."""
    k = 1025 if dtype == "f32" else 2049
    _check_forward(33, 2027, k, 17, LOG[32, 128, True], dtype, BI, -k % 64 if pad is None else pad, seed=3)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,pad", [(600, 0), (640, 0), (601, 3), (2500, 0)])
def test_one_token_of_many_heads(k, pad, dtype):
    _check_forward(520, 1, k, k - 1, LOG[32, 128, False], dtype, CAUSAL, pad)
    _check_forward(520, 3, k, k - 3, LOG[32, 128, False], dtype, CAUSAL, pad, 16)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch,heads,q,k,start,pad", [
    (2, 16, 512, 1531, 700, 0), (3, 16, 509, 1531, 0, 0), (2, 17, 515, 1536, 1021, 3), (2, 16, 1021, 640, 0, 0), (1, 40, 700, 2049, 1349, 0),   # tiles of 32 rows
    (1, 16, 250, 1531, 700, 0), (1, 12, 333, 1400, 1, 1),                                                                                   # of 16 or 32
    (1, 4, 333, 1100, 500, 0), (1, 1, 1000, 1000, 0, 0),                                                                                     # of 8 or 16
])
def test_gradients_of_a_causal_bias(batch, heads, q, k, start, pad, dtype):
    """Hidden places hold NaN (see _check): none of it is seen, wherever the border passes through a tile."""
    _check(heads, q, k, start, LOG[32, 128, False], dtype, CAUSAL, batch, pad, seed=heads)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("flags", [0, BI])
def test_gradients_in_tiles_of_32_rows(flags, dtype):
    _check(16, 517, 1531, 600, LOG[64, 800, True] if flags else LOG[128, 300, False], dtype, flags, batch=2, seed=5)
    _check(12, 701, 2049, 0, list(range(1, 120)), dtype, flags, batch=2, pad=9, seed=6)
