"""Performance cases of the operators that a training step or an inference loop needs around the layers.

* ``lnorm``   LayerNorm of rows, with or without a residual added first; training adds its backward pass with the gradients of
              gamma and beta;
* ``relpos``  the relative position bias by buckets of offsets: as the table of a window (what the attention layer takes) or as the
              bias of a sequence's scores, with the gradient of the learned rows when training;
* ``adamw``   one AdamW step over all tensors of a model, states in 32 or 8 bits, clipped by the norm of all gradients or not.

Shapes are those of the layers here (60 and 180 channels, 64x64 patches, 8x8 to 16x16 windows, stacks of 36) and generic ones.
"""
import math

import torch

own = False   # False: the plain form below; True: the calls of the package's entry points

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
BLOCK = 256   # elements that share an exponent where states are held in 8 bits; tensors start at multiples of it
BETA1, BETA2, ADAM_EPS, LR, DECAY, SEED = 0.9, 0.999, 1e-8, 2e-4, 0.01, 20240


def _lnorm(rows, C, dtype, residual, train, pad=0):
    return dict(op="lnorm", rows=rows, C=C, dtype=dtype, residual=residual, train=train, pad=pad)


def _window(M, heads, buckets, distance, dtype):
    return dict(op="relpos", form="window", window=M, heads=heads, buckets=buckets, distance=distance, dtype=dtype, train=True,
                bidirectional=True)


def _sequence(batch, heads, q, k, start, buckets, distance, dtype, train, bidirectional=True, causal=False):
    return dict(op="relpos", form="sequence", batch=batch, heads=heads, q=q, k=k, start=start, buckets=buckets, distance=distance,
                dtype=dtype, train=train, bidirectional=bidirectional, causal=causal)


def _adamw(kind, layers, width, bits, p, g="f32", clip=True):
    return dict(op="adamw", kind=kind, layers=layers, width=width, bits=bits, p=p, g=g, clip=clip)


def listed():
    return [
        # a few tokens of a decoding step: latency
        dict(_lnorm(8, 2048, "bf16", True, False), name="lnorm_tokens_bf16"),
        # the end of a sequence of layers: 32 patches of 64x64 with 180 channels
        dict(_lnorm(32 * 64 * 64, 180, "bf16", False, True), name="lnorm_train_c180"),
        # full precision, an odd width, rows of a wider tensor
        dict(_lnorm(4099, 1531, "f32", True, True, 37), name="lnorm_train_odd_f32"),
        # a long batch of wide rows with a residual
        dict(_lnorm(32768, 4096, "bf16", True, True), name="lnorm_train_wide_bf16"),
        # the table of a 16x16 window from 31 x 31 offsets in 18 x 18 buckets, both directions: latency
        dict(_window(16, 6, 18, 14, "bf16"), name="relpos_window16"),
        # one new token against a cache
        dict(_sequence(1, 32, 1, 8190, 8189, 32, 128, "bf16", False, False, True), name="relpos_one_token"),
        # causal training of odd lengths with a prefix, full precision
        dict(_sequence(2, 12, 1021, 1531, 510, 32, 128, "f32", True, False, True), name="relpos_train_causal_f32"),
        # an encoder's bias for long sequences, shared by a batch
        dict(_sequence(2, 16, 4096, 4096, 0, 32, 128, "bf16", True), name="relpos_train_4096"),
        # one whole layer in full precision: latency
        dict(_adamw("swin", 1, 60, 32, "f32", clip=False), name="adamw_one_layer_f32"),
        # 36 layers of 60 channels, bf16 parameters with an fp32 copy: 468 small tensors
        dict(_adamw("swin", 36, 60, 32, "bf16+f32"), name="adamw_stack36_c60"),
        # 36 layers of 180 channels, states in 8 bits, no fp32 copy
        dict(_adamw("swin", 36, 180, 8, "bf16"), name="adamw_stack36_c180_8bit"),
        # four dense blocks of 2048 channels (201 M parameters), states in 8 bits beside an fp32 copy
        dict(_adamw("dense", 4, 2048, 8, "bf16+f32", "bf16"), name="adamw_dense_8bit"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("lnorm", "relpos", "adamw"))
    dtype = rng.choice(("f32", "bf16", "bf16"))
    if op == "lnorm":
        C = _log_int(rng, 32, 8192)
        if rng.random() < 0.5:
            C = max(8, C // 8 * 8)
        train = rng.random() < 0.6
        rows = _log_int(rng, 1, 32768 * 4096 // (2 * C if dtype == "f32" else C))
        return _lnorm(rows, C, dtype, rng.random() < 0.5, train, rng.choice((0, 0, 8, 5)))
    if op == "relpos":
        if rng.random() < 0.2:
            return _window(rng.randint(4, 32), rng.randint(1, 16), 2 * rng.randint(2, 24), rng.randint(16, 64), dtype)
        bidirectional = rng.random() < 0.5
        buckets, distance = 2 * rng.randint(4, 64), _log_int(rng, 65, 2048)
        heads = rng.randint(1, 24)
        if rng.random() < 0.25:
            k = _log_int(rng, 1, 65536)
            return _sequence(1, heads, 1, k, k - 1, buckets, distance, dtype, False, bidirectional, True)
        batch, q, k = rng.randint(1, 4), _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
        while (batch + 1) * heads * q * k * (2 if dtype == "f32" else 1) > 3 * 16 * 4096 * 4096:
            heads = max(1, heads // 2)
            batch = max(1, batch - 1)
        start = max(0, k - q) if rng.random() < 0.5 else 0
        return _sequence(batch, heads, q, k, start, buckets, distance, dtype, rng.random() < 0.7, bidirectional,
                         not bidirectional and rng.random() < 0.7)
    bits = rng.choice((8, 32))
    p = rng.choice(("f32", "bf16", "bf16+f32"))
    if rng.random() < 0.5:
        return _adamw("swin", rng.randint(1, 36), rng.randrange(60, 241, 12), bits, p, "f32", rng.random() < 0.7)
    return _adamw("dense", rng.randint(1, 4), _log_int(rng, 64, 2048 if bits == 8 else 1600), bits, p, rng.choice(("f32", "bf16")), rng.random() < 0.7)


def _edges(buckets, distance, bidirectional):
    """Bucket n begins at the distance edges[n - 1]: single distances up to half of a side's buckets, then even steps of the logarithm
    up to `distance`.  In whole numbers, so that no border depends on a rounding."""
    side = buckets // 2 if bidirectional else buckets
    exact = side // 2
    out, n = list(range(1, exact + 1)), side - exact
    for k in range(1, n):
        r = out[-1]
        while r ** n * exact ** k < distance ** k * exact ** n:
            r += 1
        out.append(r)
    return out


def _tensors(case):
    """Shapes of a model's tensors: first those that decay, then the others."""
    w = case["width"]
    if case["kind"] == "swin":   # one layer with 6 heads in 2 groups, 8x8 windows and an MLP of twice the width
        decay, rest = [(2, 3 * w // 2, w // 2), (w, w), (2 * w, w), (w, 2 * w)], [(2, 3 * w // 2), (w,), (225, 6), (2 * w,)] + [(w,)] * 5
    else:
        decay, rest = [(3 * w, w), (w, w), (4 * w, w), (w, 4 * w)], [(3 * w,), (w,), (4 * w,)] + [(w,)] * 5
    return decay * case["layers"], rest * case["layers"]


def _ceil(n, m):
    return -(-n // m) * m


def _randn(shape, gen, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    s = {"case": case}
    if case["op"] == "lnorm":
        t, rows, C, ld = TYPES[case["dtype"]], case["rows"], case["C"], case["C"] + case["pad"]
        s["x"] = _randn((rows, ld), gen, t)[:, :C]
        s["gamma"] = (1 + 0.1 * torch.randn(C, generator=gen, device=DEVICE)).to(t)
        s["beta"] = _randn((C,), gen, t, 0.1)
        s["residual"] = _randn((rows, C), gen, t) if case["residual"] else None
        s["dy"] = _randn((rows, C), gen, t) if case["train"] else None
        s["dsum"] = _randn((rows, C), gen, t) if case["train"] and case["residual"] else None
    elif case["op"] == "relpos":
        t, heads = TYPES[case["dtype"]], case["heads"]
        s["edges"] = _edges(case["buckets"], case["distance"], case["bidirectional"])
        s["borders"] = torch.tensor(s["edges"], device=DEVICE)
        side = (len(s["edges"]) + 1) * (2 if case["bidirectional"] else 1)
        if case["form"] == "window":
            offsets = (2 * case["window"] - 1) ** 2
            s["table"] = _randn((side * side, heads), gen, t, 0.02)
            s["dout"] = _randn((offsets, heads), gen, torch.float32)
        else:
            s["table"] = _randn((side, heads), gen, t, 0.5)
            s["dout"] = _randn((case["batch"], heads, case["q"], case["k"]), gen, t, 0.01) if case["train"] else None
    else:
        decay, rest = _tensors(case)
        s["shapes"], s["offsets"], at = decay + rest, [], 0
        for i, shape in enumerate(s["shapes"]):
            if i == len(decay):
                s["decayed"] = at   # elements before it decay
            s["offsets"].append(at)
            at += _ceil(math.prod(shape), BLOCK)
        sizes = [math.prod(shape) for shape in s["shapes"]]
        # every tensor in its place of one range of memory, zeros up to the next tensor's start
        ends = torch.tensor([o + n for o, n in zip(s["offsets"], sizes)], device=DEVICE)
        span = torch.tensor([_ceil(n, BLOCK) for n in sizes], device=DEVICE)
        live = torch.arange(at, device=DEVICE) < torch.repeat_interleave(ends, span, output_size=at)
        level = torch.exp(torch.randn(len(sizes), generator=gen, device=DEVICE) * 1.5 - 6)   # gradients of tensors differ in size
        level = torch.repeat_interleave(level, span, output_size=at) * live
        s["p"] = torch.randn(at, generator=gen, device=DEVICE) * 0.02 * live
        s["master"] = None
        if case["p"] == "bf16+f32":
            s["master"] = s["p"]
        s["p"] = s["p"].to(TYPES[case["p"][:4]] if case["p"] != "f32" else torch.float32)
        s["g"] = (torch.randn(at, generator=gen, device=DEVICE) * level).to(TYPES[case["g"]])
        s["m"] = torch.randn(at, generator=gen, device=DEVICE) * level * 0.3
        s["v"] = level * level * (0.2 + torch.rand(at, generator=gen, device=DEVICE))
        if case["bits"] == 8:
            noise = torch.full((at,), 32768, dtype=torch.int32, device=DEVICE)
            s["m"], s["m_exp"] = _encode(s["m"], noise, 127)
            s["v"], s["v_exp"] = _encode(s["v"], noise, 255)
        s["step"] = torch.tensor([seed % 3000], dtype=torch.int64, device=DEVICE)
        s["max_norm"] = 1.0
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------------------

def _lnorm_plain(s):
    case, x, t = s["case"], s["x"], s["x"].dtype
    out = {}
    u = x.float()
    if case["residual"]:
        out["sum"] = (u + s["residual"].float()).to(t)
        u = out["sum"].float()
    C = case["C"]
    d = u - u.sum(1, keepdim=True) / C
    rstd = torch.rsqrt((d * d).sum(1, keepdim=True) / C + EPS)
    xh = d * rstd
    out["y"] = (xh * s["gamma"].float() + s["beta"].float()).to(t)
    if case["train"]:
        dy = s["dy"].float()
        g = dy * s["gamma"].float()
        dx = rstd * (g - g.sum(1, keepdim=True) / C - xh * ((g * xh).sum(1, keepdim=True) / C))
        if case["residual"]:
            dx = dx + s["dsum"].float()
        out["dx"], out["dgamma"], out["dbeta"] = dx.to(t), (dy * xh).sum(0), dy.sum(0)
    return out


def _bucket(r, s):
    """Buckets of offsets r = key - query, whole numbers."""
    if not s["case"]["bidirectional"]:
        return ((-r)[:, None] >= s["borders"]).sum(1)
    return (r.abs()[:, None] >= s["borders"]).sum(1) + (r > 0) * (len(s["edges"]) + 1)


def _window_rows(s):
    M = s["case"]["window"]
    b = _bucket(-torch.arange(1 - M, M, device=DEVICE), s)   # a table goes by query - key
    return (b[:, None] * 2 * (len(s["edges"]) + 1) + b[None, :]).reshape(-1)


def _relpos_plain(s):
    case, t = s["case"], s["table"].dtype
    rows, heads = s["table"].shape
    if case["form"] == "window":
        at = _window_rows(s)
        pick = (at[None, :] == torch.arange(rows, device=DEVICE)[:, None]).float()
        return {"out": s["table"][at], "dtable": pick @ s["dout"]}
    q, k, start = case["q"], case["k"], case["start"]
    r = torch.arange(1 - q, k, device=DEVICE) - start        # the offsets of the diagonals
    b = _bucket(r, s)
    by_offset = s["table"][b].t()
    if case["causal"]:
        by_offset = torch.where(r > 0, -math.inf, by_offset)
    at = torch.arange(k, device=DEVICE)[None, :] - torch.arange(q, device=DEVICE)[:, None] + (q - 1)
    out = {"out": by_offset[:, at]}
    if case["train"]:
        d = _diagonals(s["dout"], q, k)
        if case["causal"]:
            d = torch.where(r > 0, 0.0, d)
        pick = (b[:, None] == torch.arange(rows, device=DEVICE)[None, :]).float()
        out["dtable"] = (d @ pick).t()
    return out


def _diagonals(dout, q, k):
    """[heads, q + k - 1]: sums over the batch and along the diagonals key - query = const, from 1 - q on."""
    d = dout.float().sum(0)
    heads = d.shape[0]
    # rows of q + k places read as rows of q + k - 1: row i starts i places further right, so with the rows in reverse order
    # the diagonals stand below each other
    d = torch.nn.functional.pad(d.flip(1), (0, q)).reshape(heads, -1)[:, : q * (q + k - 1)]
    return d.reshape(heads, q, q + k - 1).sum(1)


def _mix(x):
    """32 bits into 32 bits, held in 64."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B9) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _noise(s, t):
    """The random 16-bit numbers of step t for every element: for m, for v and for a bf16 parameter."""
    n = s["p"].numel()   # below 2^32: the upper half of an element's number is 0
    key = _mix(_mix((SEED >> 32) ^ 0x510E527F) ^ (SEED & 0xFFFFFFFF))
    key = _mix(key ^ (t >> 32))
    key = _mix(key ^ (t & 0xFFFFFFFF))
    key = _mix(key ^ 0)
    h = _mix(torch.arange(n, device=DEVICE) ^ key)
    return (h & 0xFFFF).int(), (h >> 16).int(), (_mix(h ^ 0xBB67AE85) & 0xFFFF).int()


def _encode(x, noise, top):
    """fp32 -> 8 bits: blocks share the exponent E of their largest magnitude; a magnitude is rounded up or down to 3 bits behind the
    leading one with the probability of its remainder (`noise` against the next 16 bits) and counted down from code `top`,
    which stands for 2^(E + 1).  Below code 1 there is 0, or code 1 for second moments (top = 255: no sign)."""
    bits = x.view(torch.int32).view(-1, BLOCK)
    sign, bits = bits < 0, bits & 0x7FFFFFFF
    e = bits.amax(1, keepdim=True) >> 23
    held = (bits + (noise.view(-1, BLOCK) << 4)) >> 20
    first = (e + 1) * 8 - top
    if top == 127:
        code = torch.where(held > 0, torch.clamp(held - first, min=0), 0)
    else:
        code = torch.where(bits > 0, torch.clamp(torch.clamp(held, min=1) - first, min=1), 0)
    code = torch.minimum(code, top - (e == 254).int())
    if top == 127:
        code = code + 128 * (sign & (code > 0))
    return torch.where(e == 255, 0, code).to(torch.uint8).reshape(-1), e.reshape(-1).to(torch.uint8)


def _decode(code, e, top):
    code, e = code.view(-1, BLOCK).int(), e.int()[:, None]
    size = code & 127 if top == 127 else code
    bits = torch.clamp((e + 1) * 8 - top + size, min=1) << 20
    x = torch.where(size > 0, bits, 0).view(torch.float32)
    if top == 127:
        x = torch.where(code > 127, -x, x)
    return torch.where(e == 255, math.nan, x).reshape(-1)


def _adamw_plain(s):
    case = s["case"]
    s["step"] += 1
    t = s["step"]
    g = s["g"].float()
    out = {"step": t}
    if case["clip"]:
        out["norm"] = (g * g).sum(dtype=torch.float64).sqrt().float()
        g = g * torch.where(out["norm"] > s["max_norm"], s["max_norm"] / out["norm"], 1.0)
    eight = case["bits"] == 8
    m = _decode(s["m"], s["m_exp"], 127) if eight else s["m"]
    v = _decode(s["v"], s["v_exp"], 255) if eight else s["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    by = t.double()
    c1, c2 = (1 - torch.pow(BETA1, by)).float(), (1 - torch.pow(BETA2, by)).float()
    p = (s["p"] if s["master"] is None else s["master"]).float()
    p = torch.cat([p[: s["decayed"]] * (1 - LR * DECAY), p[s["decayed"]:]])
    p = p - LR / c1 * m / (v.sqrt() / c2.sqrt() + ADAM_EPS)
    noisy = case["p"] == "bf16"
    if eight or noisy:
        for_m, for_v, for_p = _noise(s, t)
    if s["master"] is not None:
        s["master"].copy_(p)
        out["master"] = s["master"]
    if noisy:   # nothing else holds the parameter: rounded up or down with the probability of its remainder
        p = ((p.view(torch.int32) + for_p) & -65536).view(torch.float32)
    s["p"].copy_(p)
    out["p"] = s["p"]
    if eight:
        c, e = _encode(m, for_m, 127)
        s["m"].copy_(c), s["m_exp"].copy_(e)
        c, e = _encode(v, for_v, 255)
        s["v"].copy_(c), s["v_exp"].copy_(e)
        # 4 significant bits: bf16 holds them whole
        out["m"], out["v"] = _decode(s["m"], s["m_exp"], 127).bfloat16(), _decode(s["v"], s["v_exp"], 255).bfloat16()
    else:
        s["m"].copy_(m), s["v"].copy_(v)
        out["m"], out["v"] = s["m"], s["v"]
    return out


# ---- the package's entry points --------------------------------------------------------------------------------------------------

def _lnorm_own(s):
    from paper_2409_06206_amd import lnorm
    case, x = s["case"], s["x"]
    if "desc" not in s:
        s["desc"] = lnorm.make_desc(case["rows"], case["C"], case["dtype"], EPS, x_stride=x.stride(0))
        new = lambda: torch.empty(case["rows"], case["C"], dtype=x.dtype, device=DEVICE)  # noqa: E731
        s["y"], s["sum"], s["dx"] = new(), new() if case["residual"] else None, new() if case["train"] else None
        s["dgamma"], s["dbeta"] = (torch.empty(case["C"], device=DEVICE) for _ in range(2))
        if case["residual"]:   # the backward pass reads the stored sum, whose rows lie close
            s["desc_sum"] = lnorm.make_desc(case["rows"], case["C"], case["dtype"], EPS)
        s["ws"] = torch.empty(lnorm.lnorm_query_bytes(s["desc"]), dtype=torch.uint8, device=DEVICE)
    lnorm.lnorm_forward(s["desc"], x, s["residual"], s["gamma"], s["beta"], s["y"], s["sum"])
    out = {"y": s["y"]}
    if case["residual"]:
        out["sum"] = s["sum"]
    if case["train"]:
        u, desc = (s["sum"], s["desc_sum"]) if case["residual"] else (x, s["desc"])
        lnorm.lnorm_backward(desc, u, s["dy"], s["gamma"], s["dsum"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        out.update(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    return out


def _relpos_own(s):
    from paper_2409_06206_amd import relpos
    case = s["case"]
    if "desc" not in s:
        edges = relpos.relpos_log_edges(case["buckets"], case["distance"], case["bidirectional"])
        flags = (relpos.RELPOS_BIDIRECTIONAL if case["bidirectional"] else 0) | (relpos.RELPOS_CAUSAL if case.get("causal") else 0)
        if case["form"] == "window":
            s["desc"] = relpos.make_desc(case["heads"], edges, case["dtype"], flags, window=case["window"])
            shape = s["dout"].shape
        else:
            s["desc"] = relpos.make_desc(case["heads"], edges, case["dtype"], flags, q_len=case["q"], k_len=case["k"],
                                         q_start=case["start"], batch=case["batch"])
            shape = (case["heads"], case["q"], case["k"])
        s["out"] = torch.empty(shape, dtype=s["table"].dtype, device=DEVICE)
        s["dtable"] = torch.empty(s["table"].shape, device=DEVICE)
        s["ws"] = torch.empty(relpos.relpos_query_bytes(s["desc"]), dtype=torch.uint8, device=DEVICE)
    relpos.relpos_forward(s["desc"], s["table"], s["out"])
    if not case["train"]:
        return {"out": s["out"]}
    relpos.relpos_backward(s["desc"], s["dout"], s["dtable"], s["ws"])
    return {"out": s["out"], "dtable": s["dtable"]}


def _adamw_own(s):
    from paper_2409_06206_amd import adamw
    case, eight = s["case"], s["case"]["bits"] == 8
    if "plan" not in s:
        desc = adamw.make_desc(BETA1, BETA2, ADAM_EPS, case["bits"], seed=SEED)
        tensors = []
        for shape, at in zip(s["shapes"], s["offsets"]):
            n = math.prod(shape)
            part = {k: s[k][at: at + n] for k in ("p", "g", "m", "v")}
            if s["master"] is not None:
                part["master"] = s["master"][at: at + n]
            if eight:
                part.update({k: s[k][at // BLOCK: _ceil(at + n, BLOCK) // BLOCK] for k in ("m_exp", "v_exp")})
            tensors.append(dict(part, weight_decay=DECAY if at < s["decayed"] else 0.0))
        s["plan_buffer"] = torch.empty(adamw.adamw_query_bytes(desc, tensors), dtype=torch.uint8, device=DEVICE)
        s["plan"] = adamw.adamw_plan(desc, tensors, s["plan_buffer"])
        s["norm"] = torch.empty((), device=DEVICE)
        if eight:
            s["m_out"], s["v_out"] = (torch.empty(s["p"].numel(), dtype=torch.bfloat16, device=DEVICE) for _ in range(2))
    out = {"step": s["step"]}
    if case["clip"]:
        adamw.adamw_norm(s["plan"], s["norm"])
        adamw.adamw_step(s["plan"], s["step"], LR, norm=s["norm"], max_norm=s["max_norm"])
        out["norm"] = s["norm"]
    else:
        adamw.adamw_step(s["plan"], s["step"], LR)
    if s["master"] is not None:
        out["master"] = s["master"]
    out["p"] = s["p"]
    if eight:
        adamw.adamw_unpack(s["plan"], s["m_out"], s["v_out"])
        out["m"], out["v"] = s["m_out"], s["v_out"]
    else:
        out["m"], out["v"] = s["m"], s["v"]
    return out


def run(state):
    if own:
        return {"lnorm": _lnorm_own, "relpos": _relpos_own, "adamw": _adamw_own}[state["case"]["op"]](state)
    return {"lnorm": _lnorm_plain, "relpos": _relpos_plain, "adamw": _adamw_plain}[state["case"]["op"]](state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------------

def _lnorm_exact(s):
    case, t = s["case"], s["x"].dtype
    u = s["x"].double()
    out = {}
    if case["residual"]:
        u = (u + s["residual"].double()).to(t).double()   # what is stored is what is normalised
        out["sum"] = u
    var, mean = torch.var_mean(u, dim=1, correction=0, keepdim=True)
    xh = (u - mean) / (var + EPS).sqrt()
    out["y"] = s["beta"].double() + s["gamma"].double() * xh
    if case["train"]:
        dy = s["dy"].double()
        out["dgamma"], out["dbeta"] = torch.sum(dy * xh, 0), torch.sum(dy, 0)
        dxh = dy * s["gamma"].double()
        # through xh = (u - mean) / sqrt(var + eps): d mean, then d var
        dx = (dxh - dxh.mean(1, keepdim=True) - xh * (dxh * xh).mean(1, keepdim=True)) / (var + EPS).sqrt()
        out["dx"] = dx + s["dsum"].double() if case["residual"] else dx
    return out


def _bucket_of(r, s):
    """One offset's bucket."""
    if s["case"]["bidirectional"]:
        return sum(abs(r) >= e for e in s["edges"]) + (len(s["edges"]) + 1 if r > 0 else 0)
    return sum(-r >= e for e in s["edges"])


def _relpos_exact(s):
    case, table = s["case"], s["table"].double()
    if case["form"] == "window":
        M, side = case["window"], 2 * (len(s["edges"]) + 1)
        at = [_bucket_of(-dr, s) * side + _bucket_of(-dc, s) for dr in range(1 - M, M) for dc in range(1 - M, M)]
        out = torch.stack([table[b] for b in at])
        d = torch.zeros_like(table)
        for n, b in enumerate(at):
            d[b] += s["dout"][n].double()
        return {"out": out, "dtable": d}
    q, k, start = case["q"], case["k"], case["start"]
    of = {r: _bucket_of(r, s) for r in range(1 - q - start, k - start)}
    by = torch.tensor([of[r] for r in sorted(of)], device=DEVICE)
    keys, queries = torch.arange(k, device=DEVICE), torch.arange(q, device=DEVICE) + start
    r = keys[None, :] - queries[:, None]
    b = by[r + (q - 1 + start)]
    hidden = (r > 0) if case["causal"] else torch.zeros_like(r, dtype=torch.bool)
    out = torch.empty(case["heads"], q, k, dtype=torch.float64, device=DEVICE)
    for h in range(case["heads"]):
        out[h] = table[:, h][b].masked_fill(hidden, -math.inf)
    res = {"out": out}
    if case["train"]:
        d = torch.zeros_like(table)
        for h in range(case["heads"]):
            both = s["dout"][:, h].double().sum(0).masked_fill(hidden, 0.0)
            for n in range(table.shape[0]):
                d[n, h] = (both * (b == n)).sum()
        res["dtable"] = d
    return res


def _rounded(x, noise, digits):
    """|x| to `digits` bits behind the leading one: up with the probability of what is cut off."""
    f, e = torch.frexp(x.abs())
    step = torch.ldexp(torch.ones_like(f), e - 1 - digits)
    return torch.sign(x) * torch.floor(x.abs() / step + noise.double() / 65536) * step


def _held(x, noise, lowest, never_zero):
    """What 8 bits hold of x: blocks of BLOCK, nothing below 1.25 * 2^-lowest of the power of two under the block's largest magnitude."""
    y = _rounded(x, noise, 3)
    _, e = torch.frexp(x.abs().view(-1, BLOCK).amax(1, keepdim=True))
    least = 1.25 * torch.ldexp(torch.ones_like(x.view(-1, BLOCK)), (e - 1 - lowest).expand(-1, BLOCK)).reshape(-1)
    return torch.where(x == 0, 0.0, torch.where(y.abs() < least, least if never_zero else 0.0, y))


def _adamw_exact(s):
    case, t = s["case"], int(s["step"]) + 1
    g = s["g"].double()
    out = {"step": t}
    if case["clip"]:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = norm
        g = g * min(1.0, s["max_norm"] / float(norm))
    if case["bits"] == 8:
        m, v = (_decode(s[k], s[k + "_exp"], top).double() for k, top in (("m", 127), ("v", 255)))
    else:
        m, v = s["m"].double(), s["v"].double()
    m += (1 - BETA1) * (g - m)
    v += (1 - BETA2) * (g * g - v)
    p = (s["master"] if s["master"] is not None else s["p"]).double()
    p[: s["decayed"]] *= 1 - LR * DECAY
    p -= LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
    noise = _noise(s, torch.tensor(t, device=DEVICE)) if case["bits"] == 8 or case["p"] == "bf16" else None
    if s["master"] is not None:
        out["master"] = p
    out["p"] = _rounded(p, noise[2], 7) if case["p"] == "bf16" else p
    if case["bits"] == 8:
        m, v = _held(m, noise[0], 15, False), _held(v, noise[1], 31, True)
    out["m"], out["v"] = m, v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"lnorm": _lnorm_exact, "relpos": _relpos_exact, "adamw": _adamw_exact}[case["op"]](s)


def work(case):
    """Each input read once, each output written once; a few operations an element."""
    if case["op"] == "lnorm":
        n, e = case["rows"] * case["C"], 4 if case["dtype"] == "f32" else 2
        arrays = 2 + 2 * case["residual"] + 2 * case["train"] + (case["train"] and case["residual"])
        return {"bytes": n * e * arrays + case["C"] * (2 * e + 8 * case["train"]), "flops": n * (8 + 14 * case["train"])}
    if case["op"] == "relpos":
        e = 4 if case["dtype"] == "f32" else 2
        if case["form"] == "window":
            n = (2 * case["window"] - 1) ** 2 * case["heads"]
            rows = case["buckets"] ** 2 * case["heads"]
            return {"bytes": n * (e + 4) + rows * (e + 4), "flops": n}
        q, k, start = case["q"], case["k"], case["start"]
        out = case["heads"] * q * k
        seen = sum(min(k, max(0, i + start + 1)) for i in range(q)) if case["causal"] else q * k   # gradients of hidden places are not read
        read = case["batch"] * case["heads"] * seen if case["train"] else 0
        return {"bytes": (out + read) * e + case["buckets"] * case["heads"] * (e + 4 * case["train"]), "flops": out + read}
    decay, rest = _tensors(case)
    n = sum(math.prod(shape) for shape in decay + rest)
    p = {"f32": 8, "bf16": 4, "bf16+f32": 10}[case["p"]]   # the parameter read and written (beside an fp32 copy only written)
    states = 16 if case["bits"] == 32 else 4 + 4            # read and written; in 8 bits also read out, as 2 x 2 bytes
    return {"bytes": n * (p + states + (4 if case["g"] == "f32" else 2)), "flops": n * (14 + 2 * case["clip"])}
