"""The operators on group-scaled packed rows, as a program that serves or fine-tunes a language model calls them.

Rows of 4- or 8-bit values in the packed storage format (bits * i .. of word i // (32 / bits)) with one float scale, and for
unsigned values one whole zero point, for every `group` consecutive values: value = scale * (q - zero).  Kinds of case:

  roundtrip  float rows are quantised into group-scaled rows and read back
  matmul     y = x W^T with 4-bit weights W (M rows of K), for one token or many
  grad       dx = dy W, the gradient of matmul's input
  ffn        h = act(x Wg^T) * (x Wu^T), then y = h Wd^T: a feed-forward block as it is served
  back       from stored 8-bit projections: dg, du, then dx = dg Wg + du Wu
  train      the gated block's forward pass with its projections stored in 8 bits, and its backward pass

"type" is the type of every floating tensor that enters or leaves (scales are float).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SAVED = 32   # consecutive values that share a scale in the stored projections
TINY = 2.0 ** -100   # a group whose values (or range) stay below this is stored as zeros


def _case(name, kind, T, M, K, group, signed, typ, act="silu", bits=4):
    return {"name": name, "kind": kind, "T": T, "M": M, "K": K, "group": group, "signed": signed, "type": typ, "act": act,
            "bits": bits}


def listed():
    return [
        # weights of one layer on their way into 4 bits with zero points, rows that are no whole number of words
        _case("weights_u4", "roundtrip", 4096, 0, 4099, 128, False, "f32"),
        # a batch's activations put aside in 8 bits for the backward pass, and read back there
        _case("checkpoint_s8", "roundtrip", 8192, 0, 4096, 32, True, "bf16", bits=8),
        # one token, a small projection: a call bound by its launch
        _case("token_small", "matmul", 1, 512, 512, 32, True, "f16"),
        # one token, an ordinary projection
        _case("token", "matmul", 1, 4096, 4096, 128, True, "bf16"),
        # one token, the largest projection: bound by reading the weights
        _case("token_large", "matmul", 1, 16384, 8192, 128, False, "bf16"),
        # sixteen sequences decoded together
        _case("batch16", "matmul", 16, 4096, 4096, 64, False, "f16"),
        # a prompt
        _case("prompt", "matmul", 2048, 4096, 4096, 128, True, "bf16"),
        # odd sizes everywhere, 32-bit activations, the smallest groups
        _case("ragged_f32", "matmul", 77, 1013, 2051, 32, False, "f32"),
        # the feed-forward block for one token
        _case("ffn_token", "ffn", 1, 10240, 4096, 128, True, "bf16"),
        # the gradient through one projection of a short batch
        _case("grad_f16", "grad", 1024, 4096, 4096, 64, False, "f16"),
        # the backward pass alone, from projections stored earlier, odd sizes, 32-bit gradients
        _case("back_f32", "back", 333, 1511, 1003, 32, False, "f32", act="gelu"),
        # a training step of the gated block on frozen weights: the largest
        _case("train", "train", 2048, 10240, 4096, 128, True, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["roundtrip", "matmul", "matmul", "matmul", "grad", "ffn", "back", "train"])
    typ = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "train" and typ == "f32":
        typ = "bf16"
    group, signed, act = rng.choice([32, 64, 128]), rng.random() < 0.5, rng.choice(["silu", "gelu"])
    if kind == "roundtrip":
        return {k: v for k, v in _case("", kind, _log(rng, 1, 8192), 0, _log(rng, 32, 8192), group, signed, typ, act,
                                       rng.choice([4, 8])).items() if k != "name"}
    M, K = _log(rng, 256, 10240), _log(rng, 256, 8192)
    if rng.random() < 0.5:   # layers are mostly round numbers, not always
        M, K = -(-M // 64) * 64, -(-K // 64) * 64
    if kind == "matmul":
        T = rng.choice([1, 2, _log(rng, 3, 64), _log(rng, 65, 2048)])
    elif kind == "ffn":
        T = rng.choice([1, _log(rng, 2, 64)])
    else:
        T = _log(rng, 32, 2048)
    return {k: v for k, v in _case("", kind, T, M, K, group, signed, typ, act).items() if k != "name"}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _weights(case, rows, cols, gen):
    """4-bit rows as a checkpoint file holds them: words, scales, and zero points where the values are unsigned."""
    words = (cols + 7) // 8
    q = torch.randint(-2 ** 31, 2 ** 31, (rows, words), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    if cols % 8:
        q[:, -1] &= (1 << 4 * (cols % 8)) - 1   # fields behind the row's end are 0
    groups = -(-cols // case["group"])
    scale = (0.5 + torch.rand(rows, groups, generator=gen, device="cuda")) * (0.25 / math.sqrt(cols))
    zero = None if case["signed"] else torch.randint(5, 12, (rows, groups), generator=gen, device="cuda",
                                                     dtype=torch.int32).to(torch.uint8)
    return {"q": q, "scale": scale, "zero": zero, "cols": cols, "bits": 4, "group": case["group"]}


def _saved(rows, cols, gen, spread):
    """8-bit rows as the forward pass stored them."""
    q = torch.randn(rows, -(-cols // 4) * 4, generator=gen, device="cuda").mul_(40).round_().clamp_(-127, 127)
    q[:, cols:] = 0
    scale = (0.5 + torch.rand(rows, -(-cols // SAVED), generator=gen, device="cuda")) * (spread / 40)
    return {"q": q.to(torch.int8).view(torch.int32), "scale": scale, "zero": None, "cols": cols, "bits": 8, "group": SAVED}


def _activations(T, K, gen, typ, spread=1.0):
    """Normally distributed, a few columns far larger; a batch's last token is padding."""
    x = torch.randn(T, K, generator=gen, device="cuda") * spread
    x[:, ::97] *= 6.0
    if T >= 16:
        x[-1] = 0
    return x.to(TYPES[typ])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, T, M, K, typ = case["kind"], case["T"], case["M"], case["K"], case["type"]
    s = dict(case)
    if kind == "roundtrip":
        s["x"] = _activations(T, K, gen, typ, 1.0 if case["bits"] == 8 else 1.0 / math.sqrt(K))
    elif kind == "matmul":
        s["x"], s["w"] = _activations(T, K, gen, typ), _weights(case, M, K, gen)
    elif kind == "grad":
        s["dy"], s["w"] = _activations(T, M, gen, typ), _weights(case, M, K, gen)
    elif kind == "ffn":
        s["x"] = _activations(T, K, gen, typ)
        s["wg"], s["wu"], s["wd"] = _weights(case, M, K, gen), _weights(case, M, K, gen), _weights(case, K, M, gen)
    elif kind == "back":
        s["dh"], s["g"], s["u"] = _activations(T, M, gen, typ), _saved(T, M, gen, 1.0), _saved(T, M, gen, 1.0)
        s["wg"], s["wu"] = _weights(case, M, K, gen), _weights(case, M, K, gen)
    else:
        s["x"], s["dh"] = _activations(T, K, gen, typ), _activations(T, M, gen, typ)
        s["wg"], s["wu"] = _weights(case, M, K, gen), _weights(case, M, K, gen)
    return s


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _run_own(s):
    import paper_1809_10572_amd as samd
    kind = s["kind"]

    def rows(d):
        return samd.GroupRows(d["q"], d["scale"], d["zero"], d["cols"], d["bits"], d["group"])

    if kind == "roundtrip":
        r = samd.group_quantize(s["x"], s["bits"], s["signed"], s["group"])
        return {"values": samd.group_dequantize(r, s["x"].dtype), "scale": r.scale, "zero": r.zero}
    if kind == "matmul":
        return samd.group_matmul(s["x"], rows(s["w"]))
    if kind == "grad":
        return samd.group_matmul_grad(s["dy"], rows(s["w"]))
    if kind == "ffn":
        h = samd.group_gated(s["x"], rows(s["wg"]), rows(s["wu"]), s["act"])
        return {"h": h, "y": samd.group_matmul(h, rows(s["wd"]))}
    wg, wu = rows(s["wg"]), rows(s["wu"])
    if kind == "back":
        dg, du = samd.group_gated_grad(s["dh"], rows(s["g"]), rows(s["u"]), s["act"])
        return {"dg": dg, "du": du, "dx": samd.group_matmul_grad(dg, wg, du, wu)}
    h, g, u = samd.group_gated_save(s["x"], wg, wu, s["act"])
    dg, du = samd.group_gated_grad(s["dh"], g, u, s["act"])
    return {"h": h, "dg": dg, "du": du, "dx": samd.group_matmul_grad(dg, wg, du, wu)}


# ---- the plain form: elementary operations in 32 bits, each operator's results rounded once ------------------------

def _values(d):
    """The 32-bit values that group-scaled rows stand for."""
    bits, cols, group = d["bits"], d["cols"], d["group"]
    q = (d["q"].unsqueeze(-1) >> torch.arange(0, 32, bits, device="cuda", dtype=torch.int32)) & ((1 << bits) - 1)
    q = q.flatten(1)[:, :cols]
    if d["zero"] is None:
        q = q - ((q >> (bits - 1)) << bits)
    else:
        q = q - d["zero"].int().repeat_interleave(group, 1)[:, :cols]
    return q.float() * d["scale"].repeat_interleave(group, 1)[:, :cols]


def _quantised(x, bits, signed, group):
    """Whole values, scales and zero points of the rows of x (32 bits), by the operator's rule."""
    cols = x.shape[1]
    x = torch.nn.functional.pad(x, (0, -cols % group)).unflatten(1, (-1, group))
    top = 2 ** (bits - 1) - 1 if signed else 2 ** bits - 1
    if signed:
        low, span = None, x.abs().amax(2)
    else:
        low = x.amin(2).clamp(max=0)
        span = x.amax(2).clamp(min=0) - low
    inv = torch.full_like(span, top) / span
    none, bad = span < TINY, ~torch.isfinite(span)
    scale = span * torch.tensor(1 / top, dtype=torch.float32, device="cuda")
    scale = torch.where(bad, math.nan, torch.where(none, 0.0, scale))
    inv = torch.where(none | bad, 0.0, inv)
    x = torch.where(bad.unsqueeze(2), 0.0, x)
    q = torch.round(x * inv.unsqueeze(2))
    if signed:
        return q.clamp(-top, top).flatten(1)[:, :cols], scale, None
    zero = torch.where(none | bad, 0.0, torch.round(-low * inv)).clamp(0, top)
    return (q + zero.unsqueeze(2)).clamp(0, top).flatten(1)[:, :cols], scale, zero


def _through(x, bits, signed, group):
    """(values that x becomes in so many bits, scales, zero points)."""
    q, scale, zero = _quantised(x, bits, signed, group)
    cols = x.shape[1]
    if zero is not None:
        q = q - zero.repeat_interleave(group, 1)[:, :cols]
    return q * scale.repeat_interleave(group, 1)[:, :cols], scale, zero


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def run(s):
    if own:
        return _run_own(s)
    kind, act, typ = s["kind"], s["act"], TYPES[s["type"]]
    if kind == "roundtrip":
        values, scale, zero = _through(s["x"].float(), s["bits"], s["signed"], s["group"])
        return {"values": values.to(typ), "scale": scale, "zero": None if zero is None else zero.to(torch.uint8)}
    if kind == "matmul":
        return (s["x"].float() @ _values(s["w"]).t()).to(typ)
    if kind == "grad":
        return (s["dy"].float() @ _values(s["w"])).to(typ)
    wg, wu = _values(s["wg"]), _values(s["wu"])
    out = {}
    if kind == "back":
        g, u = _values(s["g"]), _values(s["u"])
    else:
        x = s["x"].float()
        g, u = x @ wg.t(), x @ wu.t()
        out["h"] = (_act(g, act)[0] * u).to(typ)
        if kind == "ffn":
            out["y"] = (out["h"].float() @ _values(s["wd"]).t()).to(typ)
            return out
        g, u = _through(g, 8, True, SAVED)[0], _through(u, 8, True, SAVED)[0]
    a, da = _act(g, act)
    dh = s["dh"].float()
    out["dg"], out["du"] = (dh * u * da).to(typ), (dh * a).to(typ)
    out["dx"] = (out["dg"].float() @ wg + out["du"].float() @ wu).to(typ)
    return out


# ---- the work that cannot be left out ------------------------------------------------------------------------------

def work(case):
    T, M, K, kind = case["T"], case["M"], case["K"], case["kind"]
    size = 4 if case["type"] == "f32" else 2

    def rows(m, k, bits=4, group=case["group"], zeros=not case["signed"]):
        return m * (-(-k // (32 // bits)) * 4 + -(-k // group) * (4 + zeros))

    if kind == "roundtrip":   # read, then written in bits, read in bits, then written
        return {"bytes": 2 * T * K * size + 2 * rows(T, K, case["bits"]), "flops": 4 * T * K}
    if kind == "matmul":
        return {"bytes": (T * K + T * M) * size + rows(M, K), "flops": 2 * T * M * K}
    if kind == "grad":
        return {"bytes": (T * K + T * M) * size + rows(M, K), "flops": 2 * T * M * K}
    if kind == "ffn":
        return {"bytes": (2 * T * K + 2 * T * M) * size + 2 * rows(M, K) + rows(K, M), "flops": 6 * T * M * K}
    saved = 2 * rows(T, M, 8, SAVED, False)
    back = {"bytes": 5 * T * M * size + T * K * size + saved + 2 * rows(M, K), "flops": 4 * T * M * K}
    if kind == "back":
        return back
    return {"bytes": back["bytes"] + (T * K + T * M) * size + saved + 2 * rows(M, K), "flops": 8 * T * M * K}


# ---- the definition in 64 bits -------------------------------------------------------------------------------------

def _exact_rows(d):
    """Group-scaled rows read byte by byte, in 64 bits."""
    raw = d["q"].contiguous().view(torch.uint8)
    if d["bits"] == 4:
        raw = torch.stack((raw % 16, raw // 16), dim=2).reshape(raw.shape[0], -1)
    v = raw[:, :d["cols"]].double()
    at = torch.div(torch.arange(d["cols"], device="cuda"), d["group"], rounding_mode="floor")
    if d["zero"] is None:
        half = 2.0 ** (d["bits"] - 1)
        v = torch.where(v >= half, v - 2 * half, v)
    else:
        v = v - d["zero"].double()[:, at]
    return v * d["scale"].double()[:, at]


def _exact_through(x, bits, signed, group):
    """x put through so many bits.  A value's whole number is fixed by its 32-bit product with the 32-bit
    reciprocal step, so both are rounded as the rule says; the scale is not."""
    T, K = x.shape
    n = -(-K // group)
    padded = torch.zeros(T, n * group, dtype=torch.float64, device="cuda")
    padded[:, :K] = x.double()
    padded = padded.view(T, n, group)
    top = float(2 ** (bits - 1) - 1 if signed else 2 ** bits - 1)
    if signed:
        low, span = torch.zeros(T, n, dtype=torch.float64, device="cuda"), padded.abs().max(2).values
    else:
        low = torch.minimum(padded.min(2).values, torch.zeros((), dtype=torch.float64, device="cuda"))
        high = torch.maximum(padded.max(2).values, torch.zeros((), dtype=torch.float64, device="cuda"))
        span = (high - low).float().double()
    live = span >= TINY
    inv = torch.where(live, top / torch.where(live, span, 1.0), 0.0).float().double()
    q = (padded * inv.unsqueeze(2)).float().double().round()
    zero = (-low * inv).float().double().round().clamp(0, top)
    q = q.clamp(-top, top) if signed else (q + zero.unsqueeze(2)).clamp(0, top) - zero.unsqueeze(2)
    scale = torch.where(live, span / top, 0.0)
    return (q * scale.unsqueeze(2)).view(T, n * group)[:, :K], scale, None if signed else zero.to(torch.uint8)


def exact(case, seed):
    s = prepare(case, seed)
    kind, typ = case["kind"], TYPES[case["type"]]
    if kind == "roundtrip":
        values, scale, zero = _exact_through(s["x"], case["bits"], case["signed"], case["group"])
        return {"values": values, "scale": scale, "zero": zero}
    if kind == "matmul":
        return s["x"].double().mm(_exact_rows(s["w"]).t())
    if kind == "grad":
        return s["dy"].double().mm(_exact_rows(s["w"]))
    wg, wu = _exact_rows(s["wg"]), _exact_rows(s["wu"])

    def act(g):
        return g / (1 + torch.exp(-g)) if case["act"] == "silu" else 0.5 * g * torch.erfc(-g / math.sqrt(2.0))

    def slope(g):
        if case["act"] == "silu":
            e = torch.exp(-g.abs())   # the derivative is 1 minus its value at -g
            p = (1 + e + e * g.abs()) / (1 + e) ** 2
            return torch.where(g >= 0, p, 1 - p)
        return 0.5 * torch.erfc(-g / math.sqrt(2.0)) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)

    out = {}
    if kind == "back":
        g, u = _exact_rows(s["g"]), _exact_rows(s["u"])
    else:
        x = s["x"].double()
        g, u = x.mm(wg.t()), x.mm(wu.t())
        out["h"] = act(g) * u
        if kind == "ffn":   # the second projection reads h as the first operator gives it
            out["y"] = out["h"].to(typ).double().mm(_exact_rows(s["wd"]).t())
            return out
        g, u = _exact_through(g, 8, True, SAVED)[0], _exact_through(u, 8, True, SAVED)[0]
    out["dg"], out["du"] = s["dh"].double() * u * slope(g), s["dh"].double() * act(g)
    out["dx"] = out["dg"].to(typ).double().mm(wg) + out["du"].to(typ).double().mm(wu)
    return out
