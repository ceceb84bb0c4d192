"""Microscaled 4-bit floats as a compressor beside TopK, and the product of two operands of them, as cases that can be timed and compared.

The format: 32 consecutive values share one scale, a power of two, and are held as sign, two exponent bits and one mantissa bit (E2M1: 0, 0.5,
1, 1.5, 2, 3, 4, 6).  The scale is 2^(floor(log2 of the largest magnitude) - 2), at least 2^-127; values are rounded to the nearest, ties to
the even code, and end at 6 scales.

- ``step``      a worker's compression pass: d = grad - g, C(d) in blocks along every layer, g += C(d), the error of every layer; the message
                is read back as the dense values it stands for
- ``apply``     the receiving side: every sender's message into its estimator and, with ``model``, the model step over them
- ``quantize``  a matrix of tokens by features as an operand, in blocks along the tokens (``along`` 0) or the features (1), and back
- ``product``   alpha A B^T + beta out of two operands with blocks along the axis that is summed: a linear layer's weight gradient from its
                inputs and its outputs' gradients, into a layer's place in the flat gradient vector
"""
from __future__ import annotations

import math

import torch

own = False  # set by the measuring tool: the library's kernels instead of the plain forms

SHIFTS = 16  # starts of the gradient buffer that a state goes through: a training step meets new gradients every time
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ----------------------------------------------------------------------------- the models whose layers are compressed
def _mlp():
    return [784 * 128, 128, 128 * 10, 10]


def _resnet18():
    out, cin = [64 * 3 * 7 * 7, 64, 64], 64
    for stage, w in enumerate([64, 128, 256, 512]):
        for b in range(2):
            out += [w * cin * 9, w, w, w * w * 9, w, w] + ([w * cin, w, w] if b == 0 and stage > 0 else [])
            cin = w
    return out + [512 * 1000, 1000]


def _resnet50():
    out, cin = [64 * 3 * 7 * 7, 64, 64], 64
    for w, blocks in zip([64, 128, 256, 512], [3, 4, 6, 3]):
        for b in range(blocks):
            out += [w * cin, w, w, w * w * 9, w, w, 4 * w * w, 4 * w, 4 * w] + ([4 * w * cin, 4 * w, 4 * w] if b == 0 else [])
            cin = 4 * w
    return out + [2048 * 1000, 1000]


def _gpt2_small(d=768):
    block = [d, d, d * 3 * d, 3 * d, d * d, d, d, d, d * 4 * d, 4 * d, 4 * d * d, d]
    return [50257 * d, 1024 * d] + 12 * block + [d, d]


MODELS = {"mlp": _mlp(), "resnet18": _resnet18(), "resnet50": _resnet50(), "gpt2": _gpt2_small()}
MOST = 4 * sum(MODELS["gpt2"])  # elements over all workers: the largest listed case


def _layers(case):
    """Every tensor of the model, shrunk by a divisor, some elements longer where neither tensors nor workers are to start on 16 bytes."""
    return [max(1, -(-n // case["divisor"])) + case["odd"] for n in MODELS[case["model"]]]


# ----------------------------------------------------------------------------- cases
def _pass(name, kind, model, workers, dtype="f32", divisor=1, odd=0, model_step=False):
    return dict(name=name, kind=kind, model=model, workers=workers, dtype=dtype, divisor=divisor, odd=odd, model_step=model_step)


def _quantize(name, rows, cols, dtype, along, batch=1, pad=0):
    """``pad``: elements between the end of a row and the start of the next."""
    return dict(name=name, kind="quantize", rows=rows, cols=cols, dtype=dtype, along=along, batch=batch, pad=pad)


def _product(name, m, n, length, batch=1, beta=1.0, shift=0, gap=0):
    """``shift``: where the output starts in the flat vector; ``gap``: elements between the workers' outputs."""
    return dict(name=name, kind="product", m=m, n=n, length=length, batch=batch, beta=beta, shift=shift, gap=gap)


def listed():
    return [
        # the smallest sender: a small model's hook, four layers, the last one shorter than a block
        _pass("step-mlp", "step", "mlp", 1),
        # eight workers' worth of a CNN's odd tensors, back to back: nothing starts on 16 bytes and every layer ends inside a block
        _pass("step-resnet50-odd", "step", "resnet50", 2, odd=5),
        # the largest: four workers of a language model whose backward pass leaves bf16 gradients
        _pass("step-gpt2-w4-bf16", "step", "gpt2", 4, dtype="bf16"),
        # a small model's receiver
        _pass("apply-resnet18-div16", "apply", "resnet18", 1, divisor=16),
        # the server of four senders: their estimators and the model in one pass
        _pass("apply-gpt2-w4-model", "apply", "gpt2", 4, model_step=True),
        # one token's inputs of a 2048-wide layer
        _quantize("quantize-1-token", 1, 2048, "bf16", 0),
        # a ragged batch of tokens in f32, rows padded by one element
        _quantize("quantize-333x1001-f32", 333, 1001, "f32", 0, batch=4, pad=1),
        # a long batch's inputs of the 1.1 B model's wide layer
        _quantize("quantize-8192x5632", 8192, 5632, "bf16", 0),
        # one token's gradient of a square layer, added to a worker's vector
        _product("product-1-token", 2048, 2048, 1),
        # ragged in all three, four workers, at an odd place of the flat vector
        _product("product-1000x513-t333", 1000, 513, 333, batch=4, shift=3, gap=1),
        # few outputs and a long sum: the keys' projection over a long batch
        _product("product-256x2048-t8192", 256, 2048, 8192, beta=0.0),
        # the wide layer of the 1.1 B model for two workers
        _product("product-5632x2048-t4096", 5632, 2048, 4096, batch=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("step", "apply", "quantize", "product"))
    if kind in ("step", "apply"):
        model = rng.choice(tuple(MODELS))
        n = sum(MODELS[model])
        workers = min(rng.choice((1, 1, 2, 3, 4, 8)), MOST // n)
        return dict(kind=kind, model=model, workers=workers, dtype=rng.choice(("f32", "bf16", "f16")) if kind == "step" else "f32",
                    divisor=rng.choice((1, _log(rng, 1, n / 5_000))), odd=rng.choice((0, 0, 0, rng.randint(1, 33))),
                    model_step=kind == "apply" and rng.random() < 0.6)
    if kind == "quantize":
        return dict(kind=kind, rows=_log(rng, 1, 8192), cols=_log(rng, 1, 5632), dtype=rng.choice(tuple(DTYPES)), along=rng.choice((0, 0, 1)),
                    batch=rng.choice((1, 1, 2, 3)) if rng.random() < 0.5 else 1, pad=rng.choice((0, 0, 8, 1)))
    while True:
        m, n, length, batch = _log(rng, 16, 5632), _log(rng, 16, 5632), _log(rng, 1, 8192), rng.choice((1, 1, 2, 4))
        if batch * m * n * max(length, 64) <= 2 * 5632 * 2048 * 4096 and batch * m * n <= 2 * 5632 * 2048:
            return dict(kind=kind, m=m, n=n, length=length, batch=batch, beta=rng.choice((0.0, 1.0, 0.5)), shift=rng.choice((0, 0, 4, 3)),
                        gap=rng.choice((0, 0, 4, 1)))


# ----------------------------------------------------------------------------- the format in plain torch
def _encode(v):
    """f32 [..., blocks, 32] -> signed multiples of the scale (f32, on the E2M1 grid) and the scales' bytes (int32)."""
    byte = ((v.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp_(min=0)
    r = v * ((254 - byte) << 23).view(torch.float32)[..., None]  # a power of two: exact
    a = r.abs()
    unit = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / unit) * unit).clamp_(max=6.0)  # round() takes ties to even, and so do the codes
    return torch.copysign(q, r), byte


def _scale(byte):
    """2^(byte - 127) in f32; byte 0 is a subnormal number."""
    return torch.where(byte > 0, byte << 23, 1 << 22).view(torch.float32)


def _nibbles(q):
    """Codes 0 .. 15 of values on the E2M1 grid."""
    a = q.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    return code | (torch.signbit(q).to(torch.uint8) << 3)


def _pack(v):
    """f32 [batch, lines, length] -> codes u8 [batch, lines, 16 a block] (even entry in the low half), scales u8 [batch, tiles, tiles, 512]:
    128 lines by 4 blocks to a tile, line r and block b of it at byte (r % 32) * 16 + r // 32 * 4 + b."""
    batch, lines, length = v.shape
    nb, lt, bt = -(-length // 32), -(-lines // 128), -(-length // 128)
    q, byte = _encode(torch.nn.functional.pad(v, (0, nb * 32 - length)).view(batch, lines, nb, 32))
    c = _nibbles(q).view(batch, lines, nb * 16, 2)
    full = torch.zeros((batch, lt * 128, bt * 4), dtype=torch.uint8, device=v.device)
    full[:, :lines, :nb] = byte.to(torch.uint8)
    tiles = full.view(batch, lt, 4, 32, bt, 4).permute(0, 1, 4, 3, 2, 5).reshape(batch, lt, bt, 512)
    return c[..., 0] | (c[..., 1] << 4), tiles.contiguous()


def _unpack(codes, scales, length):
    """The f32 values [batch, lines, length] of a packed operand."""
    batch, lines, width = codes.shape
    lt, bt = scales.shape[1:3]
    c = torch.stack((codes & 15, codes >> 4), -1).view(batch, lines, width * 2)
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float32, device=codes.device)
    byte = scales.view(batch, lt, bt, 32, 4, 4).permute(0, 1, 4, 3, 2, 5).reshape(batch, lt * 128, bt * 4)[:, :lines, :width // 16]
    v = grid[c.int()].view(batch, lines, width // 16, 32) * _scale(byte.int())[..., None]
    return v.view(batch, lines, width * 2)[..., :length]


# ----------------------------------------------------------------------------- inputs
def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1009 + sum(ord(c) for c in what))
    return g


def _heavy(shape, g):
    """Student's t with three degrees of freedom: the tails of gradients."""
    z = torch.randn(shape, generator=g, device="cuda")
    chi = torch.zeros_like(z)
    chi += torch.randn(shape, generator=g, device="cuda").square_()
    chi += torch.randn(shape, generator=g, device="cuda").square_()
    chi += torch.randn(shape, generator=g, device="cuda").square_()
    return z.div_(chi.div_(3).sqrt_().clamp_(min=1e-6))


def _layer_values(layers, workers, seed, what):
    """f32 [workers, N]: heavy tails, layers of very different sizes of gradient (1e-4 to 1e-1)."""
    g = _gen(seed, what)
    size = torch.exp(torch.rand(len(layers), generator=g, device="cuda") * math.log(1e3) + math.log(1e-4))
    size = torch.repeat_interleave(size, torch.tensor(layers, device="cuda"))
    out = torch.empty((workers, sum(layers)), device="cuda")
    for w in range(workers):
        torch.mul(_heavy(sum(layers), g), size, out=out[w])
    return out


def _plan(layers):
    """Where the blocks of a worker's message come from: the first and the last element of each, and its layer."""
    n = torch.tensor(layers, device="cuda")
    blocks = (n + 31) // 32
    layer = torch.repeat_interleave(torch.arange(len(layers), device="cuda"), blocks)
    first_block, first = blocks.cumsum(0) - blocks, n.cumsum(0) - n
    begin = first[layer] + (torch.arange(len(layer), device="cuda") - first_block[layer]) * 32
    whole = all(x % 32 == 0 for x in layers)
    end = first[layer] + n[layer]
    at = begin[:, None] + torch.arange(32, device="cuda")
    # places of a worker's values, one behind the last for what fills a layer's last block up; and back
    gather = None if whole else torch.where(at < end[:, None], at, sum(layers)).view(-1)
    back = None if whole else (at < end[:, None]).view(-1)
    return dict(layer=layer, gather=gather, back=back)


def _by_block(v, plan):
    """[workers, N] -> [workers, blocks, 32], filled up with zeros."""
    if plan["gather"] is not None:
        v = torch.cat((v, v.new_zeros((v.shape[0], 1))), 1)[:, plan["gather"]]
    return v.view(v.shape[0], -1, 32)


def _flat(v, plan):
    v = v.reshape(v.shape[0], -1)
    return v if plan["back"] is None else v[:, plan["back"]]


def _matrix(case, seed, what, rows, cols, batch):
    """f32 [batch, rows, cols] of tokens by features: tokens and features of different sizes, a few features very large."""
    g = _gen(seed, what)
    size = torch.exp(torch.randn(cols, generator=g, device="cuda"))
    size = torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, size * 30, size)
    token = torch.exp(torch.randn((batch, rows, 1), generator=g, device="cuda") / 2)
    return torch.randn((batch, rows, cols), generator=g, device="cuda").mul_(size).mul_(token)


def prepare(case, seed):
    kind = case["kind"]
    s = dict(case=case, at=0)
    if kind in ("step", "apply"):
        layers, W = _layers(case), case["workers"]
        N = sum(layers)
        s["plan"] = _plan(layers)
        s["layers"] = len(layers)
        s["est"] = torch.zeros((W, N), device="cuda")
        values = _layer_values(layers, W, seed, "gradients")
        if own:
            from paper_2312_08053_b200 import binding as kb
            s["ctx"] = kb.new_context(layers, W, [1.0])
            s["msg"] = kb.Mx4Message(s["ctx"])
        if kind == "step":
            flat = torch.empty(W * N + 32 * SHIFTS, dtype=DTYPES[case["dtype"]], device="cuda")
            flat[:W * N].view(W, N).copy_(values)
            flat[W * N:] = flat[:32 * SHIFTS]
            s["grads"] = [flat[32 * i:32 * i + W * N].view(W, N) for i in range(SHIFTS)]
            s["values"] = torch.empty((W, N), dtype=torch.float32 if case["dtype"] == "f32" else torch.bfloat16, device="cuda")
            return s
        # a message as it arrives: codes and scales, by worker
        q, byte = _encode(_by_block(values, s["plan"]))
        c = _nibbles(q).view(W, -1, 2)
        s["codes"], s["scales"] = c[..., 0] | (c[..., 1] << 4), byte.to(torch.uint8)
        s["weights"], s["gamma"] = [1.0 / W] * W, 0.1
        s["x"] = torch.zeros(N, device="cuda") if case["model_step"] else None
        if own:
            s["msg"].codes[:, :s["codes"].shape[1]] = s["codes"]
            s["msg"].scales[:, :s["scales"].shape[1]] = s["scales"]
        return s
    if kind == "quantize":
        rows, cols, batch = case["rows"], case["cols"], case["batch"]
        dtype = DTYPES[case["dtype"]]
        room = torch.zeros((batch, rows, cols + case["pad"]), dtype=dtype, device="cuda")
        s["x"] = room[..., :cols]
        s["x"].copy_(_matrix(case, seed, "matrix", rows, cols, batch))
        s["y"] = torch.empty((batch, rows, cols), dtype=torch.float32 if case["dtype"] == "f32" else torch.bfloat16, device="cuda")
        if own:
            from paper_2312_08053_b200 import binding as kb
            s["operand"] = kb.Mx4Operand(*((cols, rows) if case["along"] == 0 else (rows, cols)), batch=batch)
        return s
    m, n, length, batch = case["m"], case["n"], case["length"], case["batch"]
    s["a"] = _pack(_matrix(case, seed, "inputs", length, m, batch).transpose(1, 2).contiguous())
    s["b"] = _pack(_matrix(case, seed, "outputs", length, n, batch).transpose(1, 2).contiguous() * 1e-3)
    stride = m * n + case["gap"]
    flat = torch.zeros(case["shift"] + batch * stride, device="cuda")
    flat.copy_(torch.randn(flat.shape, generator=_gen(seed, "out"), device="cuda") * 1e-2)
    s["out"] = flat[case["shift"]:].view(batch, stride)[:, :m * n].view(batch, m, n)
    if own:
        from paper_2312_08053_b200 import binding as kb
        s["A"] = kb.Mx4Operand(m, length, batch=batch, codes=s["a"][0], scales=s["a"][1])
        s["B"] = kb.Mx4Operand(n, length, batch=batch, codes=s["b"][0], scales=s["b"][1])
    return s


# ----------------------------------------------------------------------------- one pass
def _run_own(s):
    from paper_2312_08053_b200 import binding as kb
    case = s["case"]
    if case["kind"] == "step":
        kb.kimad_mx4_step(s["ctx"], s["grads"][s["at"]], s["est"], s["msg"])
        kb.kimad_mx4_read(s["ctx"], s["msg"], s["values"])
        s["at"] = (s["at"] + 1) % SHIFTS
        return dict(state=s["est"], values=s["values"], err=s["msg"].err)
    if case["kind"] == "apply":
        kb.kimad_mx4_apply(s["ctx"], s["msg"], s["est"], s["x"], s["weights"], s["gamma"])
        return dict(est=s["est"], x=s["x"])
    if case["kind"] == "quantize":
        kb.kimad_mx4_quantize(s["x"], s["operand"], case["along"])
        kb.kimad_mx4_dequantize(s["operand"], s["y"], case["along"])
        return s["y"]
    kb.kimad_mx4_product(s["A"], s["B"], s["out"], alpha=0.5, beta=case["beta"])
    return s["out"]


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["kind"] == "step":
        plan = s["plan"]
        d = _by_block(s["grads"][s["at"]].float() - s["est"], plan)
        s["at"] = (s["at"] + 1) % SHIFTS
        q, byte = _encode(d)
        v = q * _scale(byte)[..., None]
        err = torch.zeros((d.shape[0], s["layers"]), dtype=torch.float64, device="cuda")
        err.index_add_(1, plan["layer"], (d - v).square().sum(-1, dtype=torch.float64))
        flat = _flat(v, plan)
        s["est"] += flat
        s["values"].copy_(flat)
        return dict(state=s["est"], values=s["values"], err=err.float())
    if case["kind"] == "apply":
        W = case["workers"]
        grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
        c = torch.stack((s["codes"] & 15, s["codes"] >> 4), -1).view(W, -1, 32)
        s["est"] += _flat(grid[c.int()] * _scale(s["scales"].int())[..., None], s["plan"])
        if s["x"] is not None:
            s["x"] -= s["gamma"] * (s["est"] * torch.tensor(s["weights"], device="cuda")[:, None]).sum(0)
        return dict(est=s["est"], x=s["x"])
    if case["kind"] == "quantize":
        rows, cols, batch = case["rows"], case["cols"], case["batch"]
        v = s["x"].float()
        v = v.transpose(1, 2) if case["along"] == 0 else v
        length = v.shape[-1]
        q, byte = _encode(torch.nn.functional.pad(v, (0, -length % 32)).reshape(batch, v.shape[1], -1, 32))
        v = (q * _scale(byte)[..., None]).view(batch, v.shape[1], -1)[..., :length]
        s["y"].copy_(v.transpose(1, 2) if case["along"] == 0 else v)
        return s["y"]
    a, b = _unpack(*s["a"], case["length"]), _unpack(*s["b"], case["length"])
    p = torch.matmul(a, b.transpose(1, 2))
    if case["beta"]:
        s["out"].mul_(case["beta"]).add_(p, alpha=0.5)
    else:
        s["out"].copy_(p * 0.5)
    return s["out"]


def work(case):
    """Inputs once, outputs once; a message (17 bytes for 32 values) is written by its sender and read by its receiver."""
    if case["kind"] in ("step", "apply"):
        N, W = sum(_layers(case)), case["workers"]
        if case["kind"] == "step":
            g, v = (4, 4) if case["dtype"] == "f32" else (2, 2)
            return {"bytes": W * N * (g + 8 + v + 17 / 32), "flops": 6 * W * N}
        return {"bytes": W * N * (8 + 17 / 32) + (8 * N if case["model_step"] else 0), "flops": (2 + 2 * case["model_step"]) * W * N}
    if case["kind"] == "quantize":
        n = case["batch"] * case["rows"] * case["cols"]
        return {"bytes": n * (8 if case["dtype"] == "f32" else 4) + n * 17 / 32, "flops": 3 * n}
    b, m, n, t = case["batch"], case["m"], case["n"], case["length"]
    return {"bytes": b * ((m + n) * t * 17 / 32 + m * n * (8 if case["beta"] else 4)), "flops": 2 * b * m * n * t}


# ----------------------------------------------------------------------------- the same from the definition, in 64 bits
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of the codes 0 .. 7


def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(v):
    """f64 [..., 32] -> the nearest multiples on the grid times the scale: the grid's magnitudes are told apart by their midpoints, and a value
    on one of them belongs to the even code beside it."""
    top = v.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(min=-127)  # frexp's mantissa is below 1: floor(log2) is its exponent less one
    a = v.abs() * _two_to(-e)
    up = torch.zeros_like(a)
    for code in range(7):
        mid = (GRID[code] + GRID[code + 1]) / 2
        over = (a >= mid) if code % 2 else (a > mid)
        up += over * (GRID[code + 1] - GRID[code])
    return torch.where(top > 0, up * _two_to(e), 0.0) * torch.sign(v)


def _exact_blocks(v, layers):
    """The values of C(v) for f64 v [N], layer by layer."""
    out, at = torch.empty_like(v), 0
    for n in layers:
        part = torch.nn.functional.pad(v[at:at + n], (0, -n % 32)).view(-1, 32)
        out[at:at + n] = _exact_values(part).view(-1)[:n]
        at += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "step":
        layers, states, values, errs = _layers(case), [], [], []
        for w in range(case["workers"]):
            d = (s["grads"][0][w].float() - s["est"][w]).double()  # the difference is a binary32 number by definition
            v = _exact_blocks(d, layers)
            errs.append(torch.stack([p.square().sum() for p in (d - v).split(layers)]))
            states.append(s["est"][w].double() + v)
            values.append(v)
        return dict(state=torch.stack(states), values=torch.stack(values), err=torch.stack(errs))
    if case["kind"] == "apply":
        layers = _layers(case)
        v = _layer_values(layers, case["workers"], seed, "gradients")
        est = torch.stack([s["est"][w].double() + _exact_blocks(v[w].double(), layers) for w in range(case["workers"])])
        x = None
        if s["x"] is not None:
            x = s["x"].double()
            for w in range(case["workers"]):
                x = x - s["gamma"] * s["weights"][w] * est[w]
        return dict(est=est, x=x)
    if case["kind"] == "quantize":
        v = s["x"].double()
        if case["along"] == 0:
            v = v.transpose(1, 2)
        length = v.shape[-1]
        q = _exact_values(torch.nn.functional.pad(v, (0, -length % 32)).unflatten(-1, (-1, 32))).flatten(-2)[..., :length]
        return q.transpose(1, 2).contiguous() if case["along"] == 0 else q
    out = []
    for i in range(case["batch"]):
        factors = []
        for what, lines, by in (("inputs", case["m"], 1.0), ("outputs", case["n"], 1e-3)):
            v = (_matrix(case, seed, what, case["length"], lines, case["batch"])[i] * by).double().t()
            factors.append(_exact_values(torch.nn.functional.pad(v, (0, -case["length"] % 32)).unflatten(-1, (-1, 32))).flatten(-2))
        out.append(0.5 * factors[0] @ factors[1].t() + case["beta"] * s["out"][i].double())
    return torch.stack(out)
