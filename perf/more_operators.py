"""What a training step of the head on an embedding needs beside its layers, and the layers in 8-bit floating point, as
measurable cases.

  linear   Y = act(X W^T + b) + R from X in its type, put into 8-bit floating point by the call, and W kept in it
  step     a training step of that layer: X and W into 8 bits (also transposed), forward, and from dY: dX, dW, db
  adamw    an AdamW step over many tensors at once, the moments held in 8 or in 32 bits; the step's moments are read out
  loss     softmax cross-entropy of rows of logits over classes, and where "grad" is set its gradient

8-bit floating point is e4m3 with a power of two for each 128 columns of a row (of W: for each 128 x 128 entries), the
smallest at which the block's largest magnitude is at most 448.  The gradient of the activation goes into 8 bits twice: in
blocks of 128 columns of a row for dX, in blocks of 128 rows of a column for dW.  A value half way between two of its 8-bit
neighbours may go to either there: what is summed from such values is returned in the activations' type.

Moments in 8 bits: 128 entries of a tensor share a power of two, the smallest at which the largest is at most 1.875; the
first moment has a sign, 4 bits of exponent and 3 of mantissa, the second 5 and 3.  They are rounded up where the bits that
are cut off and a number from a sequence in the entry's index and the step's number carry, so that the mean over the steps is
right; a second moment that is not 0 does not become 0.

GELU is the form with tanh.  Rows are vertices or vertex pairs.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ("none", "relu", "gelu", "silu")
BLOCK = 128
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.01
STEP = 1000  # steps that were taken before


# ---- cases ------------------------------------------------------------------------------


def listed():
    return [
        # One pair scored by a head that is there: latency.
        dict(name="linear_one_pair", kind="linear", rows=1, k=512, n=2048, type="bf16", act="gelu", residual=False),
        # All pairs of a large batch through a wide layer.
        dict(name="linear_131k_wide", kind="linear", rows=131_072, k=1024, n=4096, type="bf16", act="gelu", residual=False),
        # Scoring in 32 bits on a ragged batch, with odd widths.
        dict(name="linear_50k_odd", kind="linear", rows=50_021, k=260, n=1037, type="f32", act="silu", residual=True),
        # A training step of the wide layer of a head.
        dict(name="step_65k_wide", kind="step", rows=65_536, k=1024, n=2048, type="bf16", act="gelu"),
        # A training step on a ragged batch, odd widths.
        dict(name="step_20k_odd", kind="step", rows=20_011, k=132, n=517, type="f16", act="relu"),
        # A training step of a small batch, where launches count.
        dict(name="step_512", kind="step", rows=512, k=256, n=1024, type="bf16", act="silu"),
        # The parameters of a head with many layers: small tensors, odd sizes.
        dict(name="adamw_192_tensors", kind="adamw", tensors=192, entries=3_000_000, bits=8, type="bf16", copy=True),
        # An embedding of a million vertices as parameters, gradients in 32 bits.
        dict(name="adamw_134m_8bit", kind="adamw", tensors=1, entries=1 << 27, bits=8, type="f32", copy=False),
        # Moments in 32 bits, gradients and a copy of the parameters in 16.
        dict(name="adamw_50m_32bit", kind="adamw", tensors=24, entries=50_000_017, bits=32, type="bf16", copy=True),
        # One row of few classes: latency.
        dict(name="loss_one_row", kind="loss", rows=1, classes=47, type="f32", weights=False, grad=True),
        # Labels of vertices: few classes, ragged, rows weighted, some without a label, some classes left out.
        dict(name="loss_300k_odd", kind="loss", rows=300_007, classes=47, type="f32", weights=True, grad=True),
        # Pairs scored against many candidates.
        dict(name="loss_65k_4096", kind="loss", rows=65_536, classes=4096, type="bf16", weights=False, grad=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "step", "step", "step", "adamw", "adamw", "loss", "loss"])
    if kind == "adamw":
        entries = _log_int(rng, 1000, 1 << 27)
        return dict(kind=kind, tensors=_log_int(rng, 1, min(400, entries // 10)), entries=entries, bits=rng.choice([8, 8, 32]),
                    type=rng.choice(["f32", "bf16", "f16"]), copy=rng.random() < 0.5)
    if kind == "loss":
        classes = _log_int(rng, 2, 65536)
        return dict(kind=kind, rows=_log_int(rng, 1, min(1 << 20, (1 << 28) // classes)), classes=classes,
                    type=rng.choice(["f32", "bf16", "f16"]), weights=rng.random() < 0.5, grad=rng.random() < 0.8)
    k, n = _log_int(rng, 16, 2048), _log_int(rng, 16, 4096)
    limit = 1 << (39 if kind == "linear" else 37)  # products of a pass
    rows = _log_int(rng, 1 if kind == "linear" else 16, max(16, min(1 << 17, limit // (k * n))))
    case = dict(kind=kind, rows=rows, k=k, n=n, type=rng.choice(["f32", "bf16", "bf16", "f16"] if kind == "linear" else ["bf16", "f16"]),
                act=rng.choice(ACTS))
    if kind == "linear":
        case["residual"] = rng.random() < 0.5
    return case


# ---- inputs -----------------------------------------------------------------------------


def _sizes(case):
    """Sizes of the tensors, and where each begins in a flat array: at a multiple of a block."""
    r = random.Random(case["entries"] * 31 + case["tensors"])
    cuts = sorted(r.sample(range(1, case["entries"]), case["tensors"] - 1))
    sizes = [b - a for a, b in zip([0] + cuts, cuts + [case["entries"]])]
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    return sizes, starts, at


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    kind, t = case["kind"], TYPES[case["type"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    if kind in ("linear", "step"):
        rows, k, n = case["rows"], case["k"], case["n"]
        s = dict(x=normal(rows, k).to(t), b=0.1 * normal(n))
        w = normal(n, k) / math.sqrt(k)
        if kind == "linear":
            # a head's weights as they are kept: their 8 bits and a power of two for each block
            s["w"], s["w_exps"] = _to_e4m3(w, True)
            s["r"] = normal(rows, n).to(t) if case["residual"] else None
        else:
            s.update(w=w.to(t), dy=(0.02 * normal(rows, n)).to(t))
        return s
    if kind == "adamw":
        sizes, starts, total = _sizes(case)
        there = torch.zeros(total + 1, device=DEV)  # 1 where a tensor has an entry
        there[torch.tensor(starts, device=DEV)] += 1
        there.index_add_(0, torch.tensor([a + n for a, n in zip(starts, sizes)], device=DEV), -torch.ones(len(sizes), device=DEV))
        there = there[:total].cumsum(0).round_() if case["tensors"] > 1 else (torch.arange(total, device=DEV) < sizes[0]).float()
        first = torch.tensor(starts + [total], device=DEV) // BLOCK
        decay = torch.tensor([0.0 if n < 4096 else DECAY for n in sizes], device=DEV)  # none on biases and norms
        # gradients of a tensor's entries differ by orders of magnitude, and so do the moments of earlier steps
        size = torch.exp(1.5 * normal(total // BLOCK, 1) - 7).expand(-1, BLOCK).reshape(-1)
        s = dict(p=0.05 * normal(total) * there, g=(size * normal(total) * there).to(t), m=0.3 * size * normal(total) * there,
                 v=(size * normal(total)).square_() * there, decay=decay.repeat_interleave(first.diff()))
        if case["bits"] == 8:
            s["m"], s["v"] = _moment8(s["m"], 4, None), _moment8(s["v"], 5, None)
        return s
    rows, classes = case["rows"], case["classes"]
    x = 2.5 * normal(rows, classes)
    if classes > 4:
        x = torch.where(torch.rand(rows, classes, generator=g, device=DEV) < 0.05, torch.full_like(x, -math.inf), x)
    target = torch.randint(classes, (rows,), generator=g, device=DEV)
    x[torch.arange(rows, device=DEV), target] = 1.0
    target = torch.where(torch.rand(rows, generator=g, device=DEV) < 0.1, torch.full_like(target, -1), target) if rows > 8 else target
    return dict(x=x.to(t), target=target.to(torch.int32), scale=1.0 / rows,
                weight=torch.rand(rows, generator=g, device=DEV) + 0.5 if case["weights"] else None)


def prepare(case, seed):
    return dict(case=case, inputs=_inputs(case, seed), out=None, taken=0)


# ---- 8-bit formats, entry by entry ------------------------------------------------------------


def _power(most, top_bits, low):
    """The smallest e >= low with most <= top * 2^e, from the bits of a float: top = 1.75 * 2^8 (e4m3) or 1.875 (moments)."""
    part, power = torch.frexp(most)  # most = part * 2^power, part in [0.5, 1)
    top_part, top_power = math.frexp(top_bits)
    return torch.clamp(power - top_power + (part > top_part).to(power.dtype), min=low)


def _two(power, like):
    """2^power by its bits."""
    return ((power.to(torch.int32) + 127) << 23).view(torch.float32).to(like.dtype)


def _blocks(x, both):
    """x (rows x columns) padded to whole blocks, as (row blocks, rows of a block, column blocks, 128)."""
    rows, k = x.shape
    tall = BLOCK if both else 1
    x = torch.nn.functional.pad(x, (0, -k % BLOCK, 0, -rows % tall))
    return x.reshape(x.shape[0] // tall, tall, x.shape[1] // BLOCK, BLOCK)


def _scaled(x, both):
    """Blocks of x divided by their units and rounded to e4m3, in 32 bits, and the units' exponents."""
    b = _blocks(x, both)
    power = _power(b.abs().amax(dim=(1, 3), keepdim=True), 448.0, -126)
    v = b / _two(power, b)
    step = torch.clamp(torch.frexp(v.abs())[1] - 1, min=-6) - 3  # of the last bit of e4m3
    unit = _two(step, v)
    return torch.round(v / unit) * unit, power


def _values(v, power, rows, k):
    return (v * _two(power, v)).reshape(-1, v.shape[2] * BLOCK)[:rows, :k]


def _e4m3(x, both):
    """x as the values that its 8-bit form stands for."""
    return _values(*_scaled(x, both), *x.shape)


def _to_e4m3(x, both):
    """The bytes, with columns padded to whole blocks, and the exponents: four of them or a multiple in a row."""
    v, power = _scaled(x, both)
    q = v.reshape(-1, v.shape[2] * BLOCK)[:x.shape[0]].to(torch.float8_e4m3fn).contiguous()
    exps = (power[:, 0, :, 0] + 127).to(torch.uint8)
    return q, torch.nn.functional.pad(exps, (0, -exps.shape[1] % 4)).contiguous()


def _from_e4m3(q, exps, rows, k, both):
    b = _blocks(q.float(), both)
    power = exps[:, :b.shape[2]].to(torch.int32)[:, None, :, None] - 127
    return _values(b, power, rows, k)


def _moment8(x, exponent_bits, step):
    """x (flat, blocks of 128) as the values that its 8 bits stand for.  The bits of a float below the third of its mantissa
    are cut off, after the addition of 20 bits that follow from the entry's index in its tensor and the step's number
    ((index, number), or None: nothing is added)."""
    b = x.reshape(-1, BLOCK)
    power = _power(b.abs().amax(dim=1, keepdim=True), 1.875, -126 + 31)
    lowest = 2 - (1 << (exponent_bits - 1)) * 2  # exponent of the smallest number with a leading one: -14 or -30
    down = 2.0 ** (-126 - lowest)                # puts that number where floats begin to lose bits
    bits = (b.abs() / _two(power, b) * down).view(torch.int32)
    if step is not None:
        bits = bits + step.reshape(-1, BLOCK)
    bits = bits >> 20 << 20
    if exponent_bits == 5:  # what is more than nothing stays so
        bits = torch.where((b > 0) & (bits == 0), torch.full_like(bits, 1 << 20), bits)
    kept = bits.view(torch.float32) / down * _two(power, b)
    return (torch.sign(b) * kept).reshape(-1)


def _sequence(index, number, other):
    """20 bits for each index: the fractional parts of multiples of the golden ratio and of the root of 2."""
    h = (index * 2654435769 + number * 1779033703) & 0xFFFFFFFF
    return (((~h if other else h) & 0xFFFFFFFF) >> 12).to(torch.int32)


# ---- plain forms ------------------------------------------------------------------------


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _plain(state):
    case, s = state["case"], state["inputs"]
    kind, t = case["kind"], TYPES[case["type"]]
    if kind == "linear":
        w = _from_e4m3(s["w"], s["w_exps"], case["n"], case["k"], True)
        y = _act(_e4m3(s["x"].float(), False) @ w.t() + s["b"], case["act"])
        return {"y": (y if s["r"] is None else y + s["r"].float()).to(t)}
    if kind == "step":
        x, w = s["x"].float(), s["w"].float()
        w8 = _e4m3(w, True)
        z = _e4m3(x, False) @ w8.t() + s["b"]
        y, z = _act(z, case["act"]).to(t), z.to(t).float()
        dz = s["dy"].float() * _act_slope(z, case["act"])
        dx = _e4m3(dz, False) @ w8
        dw = _e4m3(dz.t().contiguous(), False) @ _e4m3(x.t().contiguous(), False).t()
        return {"y": y, "dx": dx.to(t), "dw": dw.to(t), "db": dz.sum(dim=0).to(t)}
    if kind == "adamw":
        return _plain_adamw(state)
    x, target = s["x"].float(), s["target"].long()
    most = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - most)
    total = e.sum(dim=1, keepdim=True)
    there = target >= 0
    at = torch.clamp(target, min=0)[:, None]
    weight = there.float() if s["weight"] is None else torch.where(there, s["weight"], torch.zeros_like(s["weight"]))
    loss = (torch.log(total) + most - torch.gather(x, 1, at))[:, 0]
    loss = torch.where(there, weight * loss, torch.zeros_like(loss))
    if not case["grad"]:
        return {"loss": loss}
    d = e / total
    d.scatter_add_(1, at, -torch.ones_like(total))
    return {"loss": loss, "dx": (d * (weight * s["scale"])[:, None]).to(t)}


def _plain_adamw(state):
    case, s = state["case"], state["inputs"]
    if state["out"] is None:
        sizes, starts, total = _sizes(case)
        first = torch.tensor(starts + [total], device=DEV)
        state["out"] = dict(index=torch.arange(total, device=DEV) - torch.tensor(starts, device=DEV).repeat_interleave(first.diff()))
    o = state["out"]
    state["taken"] += 1
    t = STEP + state["taken"]
    g = s["g"].float()
    m = BETA1 * s["m"] + (1 - BETA1) * g
    v = BETA2 * s["v"] + (1 - BETA2) * g * g
    far = LR / (1 - BETA1 ** t) * m / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    p = s["p"].reshape(-1, BLOCK)
    s["p"] = (p * (1 - LR * s["decay"])[:, None]).reshape(-1) - far
    if case["bits"] == 8:
        m, v = _moment8(m, 4, _sequence(o["index"], t, False)), _moment8(v, 5, _sequence(o["index"], t, True))
    s["m"], s["v"] = m, v
    held = torch.bfloat16 if case["bits"] == 8 else torch.float32  # what 8 bits stand for is exact in 16
    out = {"p": s["p"], "m": m.to(held), "v": v.to(held)}
    if case["copy"]:
        out["copy"] = s["p"].to(torch.bfloat16)
    return out


# ---- the framework's calls --------------------------------------------------------------


def _buffers(case, s):
    """What a program that calls again and again keeps: outputs, 8-bit forms, the optimiser."""
    import paper_2008_12336_amd as G

    kind, t = case["kind"], TYPES[case["type"]]
    new = lambda *shape, dtype=t: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    if kind == "linear":
        w8 = G.PackedFp8(case["n"], case["k"], 128, DEV)
        w8.q, w8.exps = s["w"], s["w_exps"]
        return dict(y=new(case["rows"], case["n"]), x8=G.PackedFp8(case["rows"], case["k"], 1, DEV), w8=w8)
    if kind == "step":
        rows, k, n = case["rows"], case["k"], case["n"]
        return dict(x8=G.PackedFp8(rows, k, 1, DEV), xt=G.PackedFp8(k, rows, 1, DEV), w8=G.PackedFp8(n, k, 128, DEV),
                    wt=G.PackedFp8(k, n, 128, DEV), z=new(rows, n),
                    out=dict(y=new(rows, n), dx=new(rows, k), dw=new(n, k), db=new(n, dtype=torch.float32)))
    if kind == "adamw":
        sizes, starts, total = _sizes(case)
        views = lambda flat: [flat[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
        copy = torch.zeros(total, dtype=torch.bfloat16, device=DEV) if case["copy"] else None
        opt = G.gosh_adamw_create(views(s["p"]), views(s["g"]), bits=case["bits"], copies=None if copy is None else views(copy),
                                  weight_decay=[0.0 if n < 4096 else DECAY for n in sizes])
        G.gosh_adamw_load(opt, s["m"], s["v"])
        held = torch.bfloat16 if case["bits"] == 8 else torch.float32
        out = dict(p=s["p"], m=new(total, dtype=held), v=new(total, dtype=held))
        if copy is not None:
            out["copy"] = copy
        return dict(opt=opt, out=out)
    out = dict(loss=new(case["rows"], dtype=torch.float32))
    if case["grad"]:
        out["dx"] = new(case["rows"], case["classes"])
    return out


def run(state):
    if not own:
        return _plain(state)
    import paper_2008_12336_amd as G

    case, s = state["case"], state["inputs"]
    if state["out"] is None:
        state["out"] = _buffers(case, s)
    o, kind = state["out"], case["kind"]
    if kind == "linear":
        G.gosh_linear_fp8(s["x"], o["x8"], o["w8"], o["y"], bias=s["b"], act=ACTS.index(case["act"]), residual=s["r"])
        return {"y": o["y"]}
    if kind == "step":
        act, out = ACTS.index(case["act"]), o["out"]
        G.gosh_pack_fp8(s["w"], o["w8"], o["wt"])
        G.gosh_pack_fp8(s["x"], o["x8"], o["xt"])
        G.gosh_linear_fp8(None, o["x8"], o["w8"], out["y"], bias=s["b"], act=act, z=o["z"])
        G.gosh_linear_fp8_backward(s["dy"], o["xt"], o["wt"], o["z"], act, dx=out["dx"], dw=out["dw"], db=out["db"])
        return {**out, "db": out["db"].to(TYPES[case["type"]])}
    if kind == "adamw":
        state["taken"] += 1
        G.gosh_adamw_step(o["opt"], lr=LR, step=STEP + state["taken"], beta1=BETA1, beta2=BETA2, eps=EPS)
        G.gosh_adamw_save(o["opt"], o["out"]["m"], o["out"]["v"])
        return o["out"]
    G.gosh_softmax_loss(s["x"], s["target"], o["loss"], o.get("dx"), weight=s["weight"], scale=s["scale"])
    return o


# ---- work -------------------------------------------------------------------------------


def work(case):
    kind, size = case["kind"], 4 if case["type"] == "f32" else 2
    if kind == "linear":
        rows, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": size * (rows * k + rows * n * (1 + case["residual"])) + n * k + 4 * n, "flops": 2 * rows * k * n}
    if kind == "step":
        rows, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": size * (2 * rows * k + 2 * n * k + 2 * rows * n) + 8 * n, "flops": 6 * rows * k * n}
    if kind == "adamw":
        entry = 8 + size + 2 * case["copy"] + (16 if case["bits"] == 32 else 4 + 4 / BLOCK + 4)  # 8 bits: read out in 16
        return {"bytes": int(entry * case["entries"]), "flops": 20 * case["entries"]}
    rows, classes = case["rows"], case["classes"]
    return {"bytes": size * rows * classes * (1 + case["grad"]) + rows * (8 + 4 * case["weights"]), "flops": 6 * rows * classes}


# ---- 64 bits ----------------------------------------------------------------------------


def _exact_act(z, act):
    """(value, slope), by sigmoids."""
    if act == "none":
        return z, z * 0 + 1
    if act == "relu":
        on = (z > 0).double()
        return z * on, on
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    c = 2 * math.sqrt(2 / math.pi)
    s = torch.sigmoid(c * z + c * 0.044715 * z ** 3)
    return z * s, s + z * s * (1 - s) * (c + 3 * c * 0.044715 * z ** 2)


def _exact_e4m3(x, both):
    """The values of the 8-bit form, block of columns by block of columns, by logarithms and a search among all 127."""
    table = torch.arange(127, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).double()
    out = torch.empty_like(x)
    two = lambda p: ((p.to(torch.int64) + 1023) << 52).view(torch.float64)  # noqa: E731  2^p
    for at in range(0, x.shape[1], BLOCK):
        part = x[:, at:at + BLOCK]
        most = part.abs().amax(dim=1, keepdim=True)
        if both:
            tall = torch.nn.functional.pad(most, (0, 0, 0, -len(most) % BLOCK)).reshape(-1, BLOCK)
            most = tall.amax(dim=1).repeat_interleave(BLOCK)[:len(most), None]
        power = torch.ceil(torch.log2(torch.where(most > 0, most, torch.full_like(most, 1e-300)) / 448))
        power = torch.clamp(torch.where(most > 448 * two(torch.clamp(power, min=-1000)), power + 1, power), min=-126)
        power = torch.where((most <= 448 * two(power - 1)) & (power > -126), power - 1, power)
        v = part.abs() / two(power)
        low = torch.clamp(torch.searchsorted(table, v.contiguous(), right=True) - 1, max=125)
        a, b = table[low], table[low + 1]
        up = (v - a > b - v) | ((v - a == b - v) & (low % 2 == 1))
        out[:, at:at + BLOCK] = torch.sign(part) * torch.where(up, b, a) * two(power)
    return out


def exact(case, seed):
    """In 64 bits, on the same inputs."""
    kind = case["kind"]
    if kind in ("linear", "step") and case["rows"] * case["k"] * case["n"] > 1 << 39:
        return None
    raw = _inputs(case, seed)
    if kind == "adamw":
        t = STEP + 1
        p, g, m, v = (raw[name].double() for name in ("p", "g", "m", "v"))
        m = m + (1 - BETA1) * (g - m)
        v = v + (1 - BETA2) * (g ** 2 - v)
        p -= LR * raw["decay"].double().repeat_interleave(BLOCK) * p
        p -= LR * (m / (1 - BETA1 ** t)) * torch.reciprocal((v / (1 - BETA2 ** t)) ** 0.5 + EPS)
        # where 8 bits go depends on the bits that 32 have: no such value
        out = {"p": p, "m": None if case["bits"] == 8 else m, "v": None if case["bits"] == 8 else v}
        if case["copy"]:
            out["copy"] = p
        return out
    if kind == "loss":
        x, target = raw["x"].double(), raw["target"].long()
        weight = (torch.ones(len(x), dtype=torch.float64, device=x.device) if raw["weight"] is None else raw["weight"].double())
        weight = weight * (target >= 0)
        mine = torch.arange(x.shape[1], device=x.device)[None, :] == target[:, None]
        lse = torch.logsumexp(x, dim=1)
        loss = weight * (lse - torch.where(mine, x, torch.zeros_like(x)).sum(dim=1))
        if not case["grad"]:
            return {"loss": loss}
        return {"loss": loss, "dx": (torch.exp(x - lse[:, None]) - mine.double()) * (weight * raw["scale"])[:, None]}
    x, b = raw["x"].double(), raw["b"].double()
    if kind == "linear":
        n, k = case["n"], case["k"]
        unit = torch.pow(2.0, raw["w_exps"].double() - 127).repeat_interleave(BLOCK, dim=0)[:n].repeat_interleave(BLOCK, dim=1)
        w = raw["w"].double()[:n, :k] * unit[:, :k]
        y = _exact_act(torch.addmm(b, _exact_e4m3(x, False), w.t()), case["act"])[0]
        return {"y": y if raw["r"] is None else y + raw["r"].double()}
    w8 = _exact_e4m3(raw["w"].double(), True)
    z = torch.addmm(b, _exact_e4m3(x, False), w8.t())
    y = _exact_act(z, case["act"])[0]
    # z as it is kept for the backward pass, in its type
    dz = raw["dy"].double() * _exact_act(z.to(TYPES[case["type"]]).double(), case["act"])[1]
    dw = torch.mm(_exact_e4m3(dz.t().contiguous(), False), _exact_e4m3(x.t().contiguous(), False).t())
    return {"y": y, "dx": torch.mm(_exact_e4m3(dz, False), w8), "dw": dw, "db": dz.sum(dim=0)}
