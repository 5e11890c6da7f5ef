"""The 8-bit training and serving path of a pruned linear layer, as a user's program calls it, and the same in plain torch.

A case is a dict of plain values with a "kind":

  linear   Y = act(X W^T + b) for serving: bf16 activations in, the weight kept in 8 bits (one scale for each block of
           128 x 128), the activations brought to 8 bits (one scale for each 128 features of a token) within the call
  train    forward and backward of that layer in a training step: the activations and the output gradient to 8 bits along
           both of their directions, then Y, dX, dW under the layer's mask, and the bias gradient
  adam     one AdamW step, W = W * Mask behind it, over every tensor of an encoder stack, moments in 8 or in 32 bits

8-bit forms.  Values are e4m3 or e5m2 (the "format"); a block's scale is a power of two, held as its exponent plus 127 in a
byte: the smallest that brings the block's largest magnitude to at most 448 (e4m3) or 57344 (e5m2).  Dividing by it is
exact, so the value's rounding (nearest, ties to even) is the only one.

8-bit moments.  m is e4m3, v is e5m2, one scale for each 128 neighbouring weights of a row.  The new moments are rounded to
one of the two neighbours with the distance as probability (random bits: a hash of seed, step, tensor and position), since
a decay by a thousandth of a value is far less than half a step of 8 bits and would be lost otherwise; a positive v is
never rounded to zero.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

E4M3, E5M2 = 0, 1
TOP = {E4M3: 8, E5M2: 15}                     # 448 = 1.75 * 2^8, 57344 = 1.75 * 2^15
DTYPE = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}
MASK32 = 0xFFFFFFFF
GOLDEN, ROOT2, ROOT3 = 0x9E3779B9, 0x6A09E667, 0xBB67AE85      # fractions of the golden ratio, of 2^(1/2) and of 3^(1/2)


def listed():
    return [
        # One token through the up-projection of a large encoder: latency is all there is.
        {"name": "linear T1 1024-4096", "kind": "linear", "tokens": 1, "n_out": 4096, "k_in": 1024, "gelu": True},
        # A short query, an odd number of tokens, the long contraction of the down-projection.
        {"name": "linear T13 4096-1024", "kind": "linear", "tokens": 13, "n_out": 1024, "k_in": 4096, "gelu": False},
        # One sentence through an attention projection.
        {"name": "linear T128 1024-1024", "kind": "linear", "tokens": 128, "n_out": 1024, "k_in": 1024, "gelu": False},
        # A batch without padding, features that fill no block of 128.
        {"name": "linear T1003 920-2128", "kind": "linear", "tokens": 1003, "n_out": 2128, "k_in": 920, "gelu": True},
        # The benchmark's number of tokens.
        {"name": "linear T4096 1024-4096", "kind": "linear", "tokens": 4096, "n_out": 4096, "k_in": 1024, "gelu": True},
        # Scoring a corpus offline.
        {"name": "linear T16384 4096-1024", "kind": "linear", "tokens": 16384, "n_out": 1024, "k_in": 4096, "gelu": False},
        # Fine-tuning on one short ragged batch, gradients in the format of the larger range.
        {"name": "train T407 480-1920 e5m2", "kind": "train", "tokens": 407, "n_out": 1920, "k_in": 480, "block": 12, "grad": E5M2},
        # A training step of the up-projection at the usual batch, three times compressed in 16-row blocks.
        {"name": "train T4096 1024-4096", "kind": "train", "tokens": 4096, "n_out": 4096, "k_in": 1024, "block": 16, "grad": E4M3},
        # Retraining one small layer: a few tensors and biases.
        {"name": "adam8 1 layer h256", "kind": "adam", "layers": 1, "hidden": 256, "bits": 8, "grad16": False, "block": 16},
        # One large layer with 32-bit moments and 32-bit gradients.
        {"name": "adam32 1 layer h1024", "kind": "adam", "layers": 1, "hidden": 1024, "bits": 32, "grad16": False, "block": 16},
        # Features that fill no block of 128, gradients as the weight gradient writes them.
        {"name": "adam8 3 layers h920", "kind": "adam", "layers": 3, "hidden": 920, "bits": 8, "grad16": True, "block": 8},
        # The whole encoder.
        {"name": "adam8 24 layers h1024", "kind": "adam", "layers": 24, "hidden": 1024, "bits": 8, "grad16": True, "block": 16},
    ]


def _log_int(rng, lo, hi, step=1):
    return min(hi, max(lo, step * int(round(lo * (hi / lo) ** rng.random() / step))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "train", "adam"])
    if kind == "linear":
        return {"kind": kind, "tokens": _log_int(rng, 1, 8192), "n_out": _log_int(rng, 64, 4096, 8), "k_in": _log_int(rng, 64, 4096, 8),
                "gelu": rng.random() < 0.5}
    if kind == "train":
        block = rng.choice([1, 8, 12, 16, 32])
        return {"kind": kind, "tokens": _log_int(rng, 16, 4096), "n_out": _log_int(rng, 96, 4032, 96), "k_in": _log_int(rng, 64, 2048, 8),
                "block": block, "grad": rng.choice([E4M3, E5M2])}
    return {"kind": kind, "layers": _log_int(rng, 1, 12), "hidden": _log_int(rng, 64, 1024, 8), "bits": rng.choice([8, 8, 32]),
            "grad16": rng.random() < 0.5, "block": rng.choice([1, 2, 4, 8])}


# ------------------------------------------------------------------------------------------ inputs
def _generator(seed, device="cuda"):
    return torch.Generator(device=device).manual_seed(seed)


def _keep(n, cols, block, rate, g):
    """Per-group flags of a pruned weight, the first row-block empty where there are several."""
    keep = (torch.rand(n // block, cols, generator=g, device="cuda") < 1.0 / rate).to(torch.uint8)
    if keep.shape[0] > 1:
        keep[0] = 0
    return keep


def _exponents(amax, fmt):
    """Byte of the smallest power of two that brings amax to the format's range."""
    frac, exp = torch.frexp(amax)                                # amax = frac 2^exp, frac in [1/2, 1)
    e = exp - 1 - TOP[fmt] + (frac > 0.875)
    return torch.where(amax > 0, (e + 127).clamp(0, 254), torch.zeros_like(e))


def _power(byte):
    """2^(byte - 127) by its bits (a power function may be off in the last place, and ties would then fall either way)."""
    byte = byte.to(torch.int32)
    return torch.where(byte > 0, byte << 23, 1 << 22).view(torch.float32)


def _blocks(x, rows, cols):
    """x as [row blocks, rows, column blocks, cols], zeros where it ends inside a block."""
    n, k = x.shape
    x = torch.nn.functional.pad(x, (0, -k % cols, 0, -n % rows))
    return x.view(x.shape[0] // rows, rows, x.shape[1] // cols, cols)


def _to_8_bits(x, rows, cols, fmt):
    """8-bit values and scale bytes of a float32 matrix, one scale for each block of rows x cols."""
    b = _blocks(x, rows, cols)
    s = _exponents(b.abs().amax(dim=(1, 3)), fmt)
    q = (b * _power(254 - s)[:, None, :, None]).to(DTYPE[fmt])
    n, k = x.shape
    return q.view(torch.uint8).reshape(b.shape[0] * rows, -1)[:n, :k], s.to(torch.uint8)


def _values(q, s, rows, cols, fmt):
    """What 8-bit values with their scales stand for."""
    n, k = q.shape
    return q.contiguous().view(DTYPE[fmt]).float() * _power(s).repeat_interleave(rows, 0)[:n].repeat_interleave(cols, 1)[:, :k]


def _padded(n, cols):
    """An 8-bit matrix of n rows whose rows begin at multiples of 16 bytes."""
    return torch.empty(n, (cols + 15) // 16 * 16, dtype=torch.uint8, device="cuda")[:, :cols]


def _shapes(case):
    h = case["hidden"]
    return [(h, h), (h, h), (h, h), (h, h), (4 * h, h), (h, 4 * h), (1, 4 * h), (1, h), (1, h), (1, h)] * case["layers"]


def prepare(case, seed):
    g = _generator(seed)
    if case["kind"] != "adam":
        t, n, k = case["tokens"], case["n_out"], case["k_in"]
        # activations with a few features that are much larger than the others, as encoders have them
        x = torch.randn(t, k, generator=g, device="cuda") * (1.0 + 15.0 * (torch.rand(k, generator=g, device="cuda") < 0.01))
        w = 0.02 * torch.randn(n, k, generator=g, device="cuda")
        block = case.get("block", 16 if n % 16 == 0 else 8)
        keep = _keep(n, k, block, 3.0, g)
        w = (w * keep.repeat_interleave(block, 0)).to(torch.bfloat16).float()
        wq, ws = _to_8_bits(w, 128, 128, E4M3)
        s = {"case": case, "X": x.to(torch.bfloat16), "bias": (0.02 * torch.randn(n, generator=g, device="cuda")).to(torch.bfloat16),
             "Wq": _padded(n, k).copy_(wq), "WS": ws, "Y": torch.empty(t, n, dtype=torch.bfloat16, device="cuda")}
        if case["kind"] == "linear":
            s["ws"] = torch.empty(t * ((k + 15) // 16 * 16 + (k + 127) // 128) + 512, dtype=torch.uint8, device="cuda")
            return s
        s["dY"] = (1e-3 * torch.randn(t, n, generator=g, device="cuda") * torch.exp(torch.randn(t, 1, generator=g, device="cuda"))).to(torch.bfloat16)
        s["keep"] = keep
        s["dX"] = torch.empty(t, k, dtype=torch.bfloat16, device="cuda")
        s["dW"] = torch.empty(n, k, dtype=torch.bfloat16, device="cuda")
        s["db"] = torch.empty(n, dtype=torch.float32, device="cuda")
        for name, cols in (("x", k), ("y", n)):                  # 8-bit forms along the features and along the tokens
            s[name + "r"], s[name + "c"] = _padded(t, cols), _padded(t, cols)
            s[name + "rs"] = torch.empty(t, (cols + 127) // 128, dtype=torch.uint8, device="cuda")
            s[name + "cs"] = torch.empty((t + 127) // 128, cols, dtype=torch.uint8, device="cuda")
        s["ws"] = torch.empty((t + 127) // 128 * n * 4 + 256, dtype=torch.uint8, device="cuda")
        return s
    # an arena for each kind of state, and the tensors as views of it, as optimisers of many tensors keep them
    shapes = _shapes(case)
    total = sum(r * c for r, c in shapes)
    blocks = sum(r * ((c + 127) // 128) for r, c in shapes)
    arenas = {"W": 0.02 * torch.randn(total, generator=g, device="cuda"),
              "g": (1e-3 * torch.randn(total, generator=g, device="cuda")).to(torch.bfloat16 if case["grad16"] else torch.float32),
              "Wb": torch.zeros(total, dtype=torch.bfloat16, device="cuda")}
    m, v = 3e-4 * torch.randn(total, generator=g, device="cuda"), 1e-6 * torch.rand(total, generator=g, device="cuda")
    if case["bits"] == 8:
        # moments as earlier steps left them: scales of their size, values all over the format
        arenas["sm"] = torch.full((blocks,), 127 - 20, dtype=torch.uint8, device="cuda")
        arenas["sv"] = torch.full((blocks,), 127 - 35, dtype=torch.uint8, device="cuda")
        arenas["m"] = (m * 2.0 ** 20).clamp(-448, 448).to(DTYPE[E4M3]).view(torch.uint8)
        arenas["v"] = (v * 2.0 ** 35).clamp(2.0 ** -16, 57344).to(DTYPE[E5M2]).view(torch.uint8)
    else:
        arenas["m"], arenas["v"] = m, v
    tensors, at, at_block = [], 0, 0
    for i, (r, c) in enumerate(shapes):
        d = {a: arenas[a][at:at + r * c].view(r, c) for a in ("W", "g", "Wb", "m", "v")}
        if case["bits"] == 8:
            kb = (c + 127) // 128
            d |= {a: arenas[a][at_block:at_block + r * kb].view(r, kb) for a in ("sm", "sv")}
            at_block += r * kb
        d["keep"] = _keep(r, c, case["block"], 3.0, g) if r > 1 else None
        d["decay"] = 0.01 if r > 1 else 0.0
        d["W"].mul_(1 if d["keep"] is None else d["keep"].repeat_interleave(case["block"], 0))
        at += r * c
        tensors.append(d)
    s = {"case": case, "arenas": arenas, "tensors": tensors, "lr": 3e-5, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "step": 1000,
         "seed": seed & 0x7FFFFFFF, "clip": torch.full((1,), 0.75, dtype=torch.float32, device="cuda")}
    if own:
        import paper_2009_08065_b200 as bsp
        s["jobs"] = bsp.make_adam_job_array([
            bsp.AdamJob(W=d["W"], grad=d["g"], m=d["m"], v=d["v"], m_scale=d.get("sm"), v_scale=d.get("sv"), keep=d["keep"], block=case["block"],
                        orient=bsp.ORIENT_C, lr=s["lr"], weight_decay=d["decay"], W_bf16=d["Wb"]) for d in tensors])
    return s


# ------------------------------------------------------------------------------------------ one pass
def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"linear": _own_linear, "train": _own_train, "adam": _own_adam}[kind](s)
    return {"linear": _plain_linear, "train": _plain_train, "adam": _plain_adam}[kind](s)


def _own_linear(s):
    import paper_2009_08065_b200 as bsp
    bsp.bsp_linear_fp8(s["Wq"], s["WS"], s["X"], s["bias"], bsp.ACT_GELU if s["case"]["gelu"] else bsp.ACT_NONE, s["Y"], s["ws"])
    return {"Y": s["Y"]}


def _own_train(s):
    import paper_2009_08065_b200 as bsp
    fmt, block = s["case"]["grad"], s["case"]["block"]
    bsp.bsp_fp8_quantize(s["X"], bsp.FP8_E4M3, s["xr"], s["xrs"], s["xc"], s["xcs"])
    bsp.bsp_linear_fp8_quantized(s["Wq"], s["WS"], s["xr"], s["xrs"], bsp.FP8_E4M3, s["bias"], bsp.ACT_NONE, s["Y"])
    bsp.bsp_fp8_quantize(s["dY"], fmt, s["yr"], s["yrs"], s["yc"], s["ycs"], s["db"], s["ws"])
    bsp.bsp_linear_fp8_backward_input(s["Wq"], s["WS"], s["yr"], s["yrs"], fmt, s["dX"])
    bsp.bsp_linear_fp8_backward_weight(s["yc"], s["ycs"], fmt, s["xc"], s["xcs"], bsp.FP8_E4M3, block, s["keep"], s["dW"])
    return {k: s[k] for k in ("Y", "dX", "dW", "db")}


def _own_adam(s):
    import paper_2009_08065_b200 as bsp
    bsp.bsp_masked_adam_step_batched(s["jobs"], s["beta1"], s["beta2"], s["eps"], s["step"], s["seed"], s["clip"])
    return _state(s)


def _state(s):
    a = s["arenas"]
    if s["case"]["bits"] == 32:
        return {k: a[k] for k in ("W", "Wb", "m", "v")}
    return {"W": a["W"], "Wb": a["Wb"], "m": a["m"].view(DTYPE[E4M3]), "v": a["v"].view(DTYPE[E5M2]), "sm": a["sm"], "sv": a["sv"]}


def _rounded(x, rows, cols, fmt):
    """x (float32) as its 8-bit form holds it."""
    return _values(*_to_8_bits(x, rows, cols, fmt), rows, cols, fmt)


def _gelu(y):
    return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))


def _plain_linear(s):
    y = _rounded(s["X"].float(), 1, 128, E4M3) @ _values(s["Wq"], s["WS"], 128, 128, E4M3).t() + s["bias"].float()
    return {"Y": (_gelu(y) if s["case"]["gelu"] else y).to(torch.bfloat16)}


def _plain_train(s):
    fmt, x, dy = s["case"]["grad"], s["X"].float(), s["dY"].float()
    w = _values(s["Wq"], s["WS"], 128, 128, E4M3)
    y = _rounded(x, 1, 128, E4M3) @ w.t() + s["bias"].float()
    dx = _rounded(dy, 1, 128, fmt) @ w
    dw = (_rounded(dy, 128, 1, fmt).t() @ _rounded(x, 128, 1, E4M3)) * s["keep"].repeat_interleave(s["case"]["block"], 0)
    return {"Y": y.to(torch.bfloat16), "dX": dx.to(torch.bfloat16), "dW": dw.to(torch.bfloat16), "db": dy.sum(0, dtype=torch.float64).float()}


def _mix(x):
    """32-bit hash, of whole numbers or of a tensor of them (64-bit integers)."""
    x = x & MASK32
    x = ((x ^ (x >> 16)) * ROOT2) & MASK32
    x = ((x ^ (x >> 15)) * ROOT3) & MASK32
    return x ^ (x >> 16)


def _stochastic(y, random, fmt):
    """Magnitudes y (float32, in the format's range) brought to one of the format's two neighbours: the bits behind the
    format's last place, with random ones (16, at their upper end) added, are cut off."""
    drop = 20 if fmt == E4M3 else 21
    low = 2.0 ** (-6 if fmt == E4M3 else -14)                    # smallest normal value; below it steps are as wide as just above
    z = torch.where(y < low, y + low, y).view(torch.int32) + (random << (drop - 16)).to(torch.int32)
    z = (z >> drop << drop).view(torch.float32)
    return torch.where(y < low, z - low, z)


def _moment(x, random, fmt):
    """New 8-bit values and scale bytes of a moment (float32 [rows, cols]), and whether v's rule holds (e5m2): no zero for a positive value."""
    b = _blocks(x, 1, 128)[:, 0]
    s = _exponents(b.abs().amax(-1), fmt)
    y = b * _power(254 - s)[..., None]
    r = _stochastic(y.abs(), _blocks(random, 1, 128)[:, 0], fmt)
    r = torch.maximum(r, 2.0 ** -16 * (b > 0)) if fmt == E5M2 else torch.copysign(r, y)
    return r.to(DTYPE[fmt]).view(torch.uint8).view(x.shape[0], -1)[:, :x.shape[1]], s.to(torch.uint8)


def _plain_adam(s):
    f = np.float32
    b1, b2, eps, lr = (float(f(s[k])) for k in ("beta1", "beta2", "eps", "lr"))
    c1, c2 = float(f(1) - f(b1)), float(f(1) - f(b2))
    i1, i2 = (float(f(1.0 / (1.0 - b ** s["step"]))) for b in (b1, b2))
    for i, d in enumerate(s["tensors"]):
        bits8, w, g = s["case"]["bits"] == 8, d["W"], d["g"].float() * s["clip"]
        m = _values(d["m"], d["sm"], 1, 128, E4M3) if bits8 else d["m"]
        v = _values(d["v"], d["sv"], 1, 128, E5M2) if bits8 else d["v"]
        # one rounding behind product and sum (in 64 bits the product is exact): the 8-bit values go by the last bit
        m = (b1 * m.double() + (c1 * g).double()).float()
        v = (b2 * v.double() + (c2 * g * g).double()).float()
        w = w - lr * ((m * i1) / (torch.sqrt(v * i2) + eps) + float(f(d["decay"])) * w)
        if d["keep"] is not None:
            w = w * d["keep"].repeat_interleave(s["case"]["block"], 0)
        d["W"].copy_(w)
        d["Wb"].copy_(w)
        if not bits8:
            d["m"].copy_(m)
            d["v"].copy_(v)
            continue
        key = _mix(s["seed"] + GOLDEN * s["step"] + ROOT3 * i)
        h = _mix(torch.arange(w.numel(), device=w.device) + key).view(w.shape)
        for name, x, random, fmt in (("m", m, h & 0xFFFF, E4M3), ("v", v, h >> 16, E5M2)):
            q, scale = _moment(x, random, fmt)
            d[name].copy_(q)
            d["s" + name].copy_(scale)
    return _state(s)


# ------------------------------------------------------------------------------------------ what cannot be done without
def work(case):
    if case["kind"] == "adam":
        shapes = _shapes(case)
        n = sum(r * c for r, c in shapes)
        groups = sum(r // case["block"] * c for r, c in shapes if r > 1)
        moments = 4 * n + 4 * sum(r * ((c + 127) // 128) for r, c in shapes) if case["bits"] == 8 else 16 * n
        return {"bytes": n * (8 + 2 + (2 if case["grad16"] else 4)) + moments + groups, "flops": 15 * n}
    t, n, k = case["tokens"], case["n_out"], case["k_in"]
    weight = n * k + ((n + 127) // 128) * ((k + 127) // 128)
    if case["kind"] == "linear":
        return {"bytes": weight + 2 * t * k + 2 * t * n + 2 * n, "flops": 2 * t * n * k}
    return {"bytes": weight + 4 * t * k + 4 * t * n + 2 * n * k + n // case["block"] * k + 6 * n, "flops": 6 * t * n * k}


# ------------------------------------------------------------------------------------------ the definition, in 64 bits
def _round_8(x, fmt):
    """Doubles to the nearest value of the format, ties to the even one."""
    mantissa, least = (3, -6) if fmt == E4M3 else (2, -14)
    steps = torch.tensor([2.0 ** (e - mantissa) for e in range(least, 17)], dtype=torch.float64, device=x.device)
    bounds = torch.tensor([2.0 ** e for e in range(least + 1, 17)], dtype=torch.float64, device=x.device)
    step = steps[torch.bucketize(x.abs(), bounds, right=True)]
    return torch.round(x / step) * step


def _scale_64(largest, fmt):
    """The smallest power of two, of those that a byte can name, that brings `largest` to the format's range."""
    powers = torch.tensor([2.0 ** e for e in range(-127, 128)], dtype=torch.float64, device=largest.device)
    return powers[torch.searchsorted(powers * (448.0 if fmt == E4M3 else 57344.0), largest.contiguous())]


def _named_64(byte):
    return torch.tensor([2.0 ** e for e in range(-127, 129)], dtype=torch.float64, device=byte.device)[byte.long()]


def _block_form_64(x, fmt, dim):
    """x in 8 bits with a scale for each 128 values along `dim`."""
    parts = []
    for part in torch.split(x.double(), 128, dim):
        scale = _scale_64(part.abs().amax(dim, keepdim=True), fmt)
        parts.append(_round_8(part / scale, fmt) * scale)
    return torch.cat(parts, dim)


def _weight_64(s):
    q, rows = s["Wq"].contiguous().view(DTYPE[E4M3]).double(), []
    scale = _named_64(s["WS"])
    for i, strip in enumerate(torch.split(q, 128, 0)):
        rows.append(torch.cat([part * scale[i, j] for j, part in enumerate(torch.split(strip, 128, 1))], 1))
    return torch.cat(rows, 0)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adam":
        return _exact_adam(s)
    w, bias = _weight_64(s), s["bias"].double()
    y = torch.matmul(_block_form_64(s["X"], E4M3, 1), w.t()) + bias
    if case["kind"] == "linear":
        return {"Y": y * torch.special.ndtr(y) if case["gelu"] else y}
    dy, fmt = s["dY"].double(), case["grad"]
    dw = torch.matmul(_block_form_64(dy, fmt, 0).t(), _block_form_64(s["X"], E4M3, 0))
    flags = s["keep"].bool()[torch.arange(case["n_out"], device="cuda") // case["block"]]
    return {"Y": y, "dX": torch.matmul(_block_form_64(dy, fmt, 1), w), "dW": torch.where(flags, dw, torch.zeros_like(dw)), "db": dy.sum(0)}


def _exact_adam(s):
    b1, b2, eps, lr, decay = (float(np.float32(x)) for x in (s["beta1"], s["beta2"], s["eps"], s["lr"], 0.01))
    out = {k: [] for k in ("W", "m", "v")}
    for d in s["tensors"]:
        g = d["g"].double() * s["clip"].double()
        m, v = d["m"], d["v"]
        if s["case"]["bits"] == 8:
            cols = m.shape[1]
            m = m.contiguous().view(DTYPE[E4M3]).double() * _named_64(d["sm"]).repeat_interleave(128, 1)[:, :cols]
            v = v.contiguous().view(DTYPE[E5M2]).double() * _named_64(d["sv"]).repeat_interleave(128, 1)[:, :cols]
        m, v = m.double() + (1 - b1) * (g - m), v.double() + (1 - b2) * (g * g - v)
        step = (m / (1 - b1 ** s["step"])) / (torch.sqrt(v / (1 - b2 ** s["step"])) + eps)
        w = d["W"].double()
        w = w - lr * (step + (decay if d["decay"] else 0.0) * w)
        if d["keep"] is not None:
            rows = torch.arange(w.shape[0], device="cuda") // s["case"]["block"]
            w = torch.where(d["keep"].bool()[rows], w, torch.zeros_like(w))
        for name, x in (("W", w), ("m", m), ("v", v)):
            out[name].append(x.reshape(-1))
    w = torch.cat(out["W"])
    if s["case"]["bits"] == 32:
        return {"W": w, "Wb": w, "m": torch.cat(out["m"]), "v": torch.cat(out["v"])}
    # rounded moments follow their random bits, which have no counterpart in 64 bits
    return {"W": w, "Wb": w, "m": None, "v": None, "sm": None, "sv": None}
