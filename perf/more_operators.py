"""A predictor's layers by role, in 8-bit integers and from 8-bit checkpoints, as a program makes the calls, for timing.

Roles have regressors of their own: a batch's rows lie role after role, as many as there are, and one
call takes every role's rows through that role's layer, or takes the gradients back. A fitted layer is
served in 8-bit integers, rows quantised as they come. A fit of many stages keeps its activations in 8 bits
between the forward and the backward pass. ``own`` chooses between the package's kernels and plain torch
operations in 32 bits (64 where a value's rounding to 8 bits is decided).
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32          # values that share a power of two in a checkpoint


def listed():
    return [
        # a scheduler tick's few hundred stages of five roles through the mid predictor's first layer, latency counts
        dict(name="grouped tick", op="grouped", n=300, groups=5, d_in=256, d_out=512, dtype="bf16", relu=True),
        # an odd shard of the wide predictor's stages, sixteen regressors, through the middle layer
        dict(name="grouped wide", op="grouped", n=262139, groups=16, d_in=1024, d_out=1024, dtype="bf16", relu=True),
        # the tiny float32 predictor (64 -> 128 -> 32), three roles
        dict(name="grouped tiny", op="grouped", n=4096, groups=3, d_in=64, d_out=128, dtype="f32", relu=True),
        # gradients of the tick's first layer
        dict(name="grouped grad tick", op="grouped_grad", n=300, groups=5, d_in=256, d_out=512, dtype="bf16", relu=False,
             want_x=False),
        # the wide predictor's middle layer, weights' and inputs' gradients
        dict(name="grouped grad wide", op="grouped_grad", n=262139, groups=16, d_in=1024, d_out=1024, dtype="bf16", relu=True,
             want_x=True),
        # a served tick in 8 bits: rows quantised and multiplied
        dict(name="int8 tick", op="int8", n=300, d_in=256, d_out=512, dtype="bf16", relu=True),
        # the wide predictor's middle layer over an odd shard
        dict(name="int8 wide", op="int8", n=262139, d_in=1024, d_out=1024, dtype="bf16", relu=True),
        # float32 features into 64 length bins, odd rows
        dict(name="int8 bins", op="int8", n=20011, d_in=512, d_out=64, dtype="f32", relu=False),
        # the wide predictor's hidden activations kept and given back
        dict(name="pack wide", op="pack", n=262139, d=1024, dtype="bf16", rectified=True),
        # a ragged batch of float32 features
        dict(name="pack features", op="pack", n=1337, d=80, dtype="f32", rectified=False),
        # the tiny predictor's first layer from kept features: weights' and biases' gradients
        dict(name="packed grad tiny", op="packed_grad", n=4096, d_in=64, d_out=128, dtype="f32", rectified=False, want_x=False),
        # the wide predictor's middle layer from its kept activations
        dict(name="packed grad wide", op="packed_grad", n=262139, d_in=1024, d_out=1024, dtype="bf16", rectified=True,
             want_x=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["grouped", "grouped_grad", "int8", "pack", "packed_grad"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    n = _log(rng, 1, 200000)
    if op == "pack":
        return dict(op=op, n=n, d=16 * _log(rng, 1, 64), dtype=dtype, rectified=rng.random() < 0.5)
    wide = 64 if dtype == "bf16" or op == "int8" else 16
    case = dict(op=op, n=n, d_in=16 * _log(rng, 1, wide), d_out=16 * _log(rng, 1, wide), dtype=dtype)
    if op == "int8":
        return dict(case, relu=rng.random() < 0.7)
    if op == "packed_grad":
        return dict(case, rectified=rng.random() < 0.6, want_x=rng.random() < 0.7)
    case = dict(case, groups=_log(rng, 1, 64), relu=rng.random() < 0.7)
    return case if op == "grouped" else dict(case, want_x=rng.random() < 0.7)


# ---------------------------------------------------------------------------------------------
# inputs, drawn on the GPU from the seed
# ---------------------------------------------------------------------------------------------

class _Rng:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device=DEV)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device=DEV)

    def rows(self, n, d, dt, f=lambda v: v):
        """[n][d] normal values, each block of rows through f."""
        x = torch.empty(n, d, device=DEV, dtype=dt)
        for a in range(0, n, 1 << 16):
            x[a:a + (1 << 16)] = f(self.normal(min(1 << 16, n - a), d)).to(dt)
        return x


def _sizes(case, seed):
    """Rows of every role: a few roles have most of them, some have one or none."""
    r = random.Random(seed * 1000003 + case["n"])
    share = [r.random() ** 3 if r.random() < 0.85 else 0.0 for _ in range(case["groups"])]
    if not sum(share):
        share[r.randrange(len(share))] = 1.0
    ends, at, total = [0], 0.0, sum(share)
    for s in share:
        at += s
        ends.append(round(case["n"] * at / total))
    ends[-1] = case["n"]
    return [b - a for a, b in zip(ends, ends[1:])]


def prepare(case, seed):
    r = _Rng(seed)
    op, n, dt = case["op"], case["n"], DTYPES[case["dtype"]]
    if op == "pack":
        # activations of rows of different size, a share of them rectified away; the spread within a row is about two decades
        gain = torch.exp(r.normal(n, 1))
        return dict(case=case, x=(r.rows(n, case["d"], torch.float32) * gain).to(dt))
    i, o = case["d_in"], case["d_out"]
    relu = torch.relu_ if op in ("grouped_grad", "packed_grad") and case.get("relu", case.get("rectified")) else lambda v: v
    x = r.rows(n, i, dt, relu)
    if op == "int8":
        w = r.normal(o, i) * i ** -0.5
        codes, scale = _codes(w)          # a served model's weights, laid out once
        return dict(case=case, x=x, w=codes.to(torch.int8), ws=scale, b=r.normal(o) * 0.1)
    gz = r.rows(n, o, dt, lambda v: v / n) if op != "grouped" else None
    if op == "packed_grad":
        codes, exponents = _pack(x, case["rectified"])
        return dict(case=case, codes=codes, exponents=exponents, w=(r.normal(o, i) * i ** -0.5).to(dt), gz=gz)
    sizes = _sizes(case, seed)
    w = (r.normal(len(sizes), o, i) * i ** -0.5).to(dt)
    offsets = torch.tensor([0] + sizes, device=DEV).cumsum(0)
    return dict(case=case, x=x, w=w, b=r.normal(len(sizes), o) * 0.1, gz=gz, sizes=sizes, offsets=offsets)


# ---------------------------------------------------------------------------------------------
# one pass: plain torch operations, or the package's kernels
# ---------------------------------------------------------------------------------------------

def _codes(x):
    """(whole numbers -127 .. 127 in 32-bit floats, scale [n]) of rows: scale the largest magnitude over 127."""
    x = x.float()
    scale = (x.abs().amax(1).double() / 127.0).float().clamp_min(2.0 ** -126)
    return torch.round(x.double() / scale.double()[:, None]).float(), scale


def _blocks(x):
    """Rows of any width as [n][blocks][BLOCK], zeros behind the last value."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK)).view(x.shape[0], -1, BLOCK)


def _power(e):
    """2^e for whole numbers e of -126 .. 127, from its bits."""
    return ((e + 127) << 23).view(torch.float32)


def _pack(x, rectified):
    """(codes [n][d], exponents [n][blocks] with 127 added): a value is code * 2^(exponent - 127). The exponent is the
    least that leaves every code of the block in 8 bits; of rectified values positive ones have codes of at least 1."""
    v = _blocks(x.float())
    if rectified:
        v = torch.relu(v)
    most = 255.0 if rectified else 127.0
    mantissa, e = torch.frexp(v.abs().amax(2))                 # mantissa in [1/2, 1)
    e = e - (8 if rectified else 7)
    e = e + (torch.round(mantissa * (most + 1)) > most).to(e.dtype)
    e = torch.where(mantissa > 0, e, -126).clamp_min(-126)
    q = torch.round(v.double() / _power(e)[:, :, None].double())
    if rectified:
        q = torch.where(v > 0, q.clamp_min(1.0), q)
    q = q.flatten(1)[:, :x.shape[1]]
    return q.to(torch.uint8 if rectified else torch.int8), (e + 127).to(torch.uint8)


def _unpack(codes, exponents):
    return (_blocks(codes.float()) * _power(exponents.int() - 127)[:, :, None]).flatten(1)[:, :codes.shape[1]]


def run(s):
    case, op = s["case"], s["case"]["op"]
    if own:
        import paper_2606_12950_amd as M
        if op == "grouped":
            return M.layer_grouped(s["x"], s["w"], s["b"], s["offsets"], relu=case["relu"])
        if op == "grouped_grad":
            return tuple(M.layer_grouped_grad(s["x"], s["w"], s["gz"], s["offsets"], relu_input=case["relu"], want_x=case["want_x"]))
        if op == "int8":
            return M.layer_int8(M.quantize_rows(s["x"]), M.Quantized(s["w"], s["ws"]), s["b"], relu=case["relu"], dtype=s["x"].dtype)
        if op == "pack":
            return M.unpack_activations(M.pack_activations(s["x"], rectified=case["rectified"]), dtype=s["x"].dtype)
        return tuple(M.layer_grad_packed(M.Packed(s["codes"], s["exponents"]), s["w"], s["gz"], relu_input=case["rectified"],
                                         want_x=case["want_x"]))
    if op == "grouped":
        y = torch.cat([x.float() @ w.float().t() + b for x, w, b in zip(s["x"].split(s["sizes"]), s["w"], s["b"])])
        return (y.relu_() if case["relu"] else y).to(s["x"].dtype)
    if op == "int8":
        q, scale = _codes(s["x"])
        y = (q @ s["w"].float().t()) * scale[:, None] * s["ws"] + s["b"]
        return (y.relu_() if case["relu"] else y).to(s["x"].dtype)
    if op == "pack":
        return _unpack(*_pack(s["x"], case["rectified"])).to(s["x"].dtype)
    masked = case["rectified"] if op == "packed_grad" else case["relu"]
    v = _unpack(s["codes"], s["exponents"]) if op == "packed_grad" else s["x"].float()
    gz, w, gx = s["gz"].float(), s["w"].float(), None
    if op == "packed_grad":
        if case["want_x"]:
            gx = gz @ w
        gw, gb = gz.t() @ v, gz.sum(0)
    else:
        parts = gz.split(s["sizes"])
        if case["want_x"]:
            gx = torch.cat([a @ b for a, b in zip(parts, w)])
        gw = torch.stack([a.t() @ b for a, b in zip(parts, v.split(s["sizes"]))])
        gb = torch.stack([a.sum(0) for a in parts])
    if case["want_x"]:
        gx = (gx * (v > 0) if masked else gx).to(s["gz"].dtype)
    return gx, gw, gb


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------

def work(case):
    e, n = 4 if case["dtype"] == "f32" else 2, case["n"]
    if case["op"] == "pack":
        d = case["d"]
        return dict(bytes=n * (2 * e * d + d + -(-d // BLOCK)), flops=4 * n * d)
    i, o = case["d_in"], case["d_out"]
    if case["op"] == "int8":
        return dict(bytes=n * (i + o) * e + i * o + 8 * o, flops=2 * n * i * o)
    groups = case.get("groups", 1)
    if case["op"] == "grouped":
        return dict(bytes=e * (n * i + n * o + groups * i * o) + 4 * groups * o, flops=2 * n * i * o)
    dx = case["want_x"]
    held = n * (i + -(-i // BLOCK)) if case["op"] == "packed_grad" else e * n * i
    return dict(bytes=held + e * (n * o + (n * i + groups * i * o if dx else 0)) + 4 * groups * (i * o + o),
                flops=2 * n * i * o * (2 if dx else 1) + n * o)


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------

def _held(codes, exponents):
    """The values of a checkpoint."""
    e = exponents.double().repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]
    return codes.double() * torch.exp2(e - 127.0)


def _held_of(v, most):
    """The values that a checkpoint of one block [n][BLOCK or fewer] holds: the least step 2^e that leaves the largest
    within the codes (of rectified values, most = 255, the positive ones)."""
    v = v.double()
    if most == 255:
        v = torch.where(v > 0, v, 0.0)
    big = torch.max(v.abs(), 1, keepdim=True).values
    e = torch.floor(torch.log2(big.clamp_min(2.0 ** -149) / most)).clamp_min(-126.0)
    e = torch.where(torch.round(big / torch.exp2(e)) > most, e + 1, e)
    e = torch.where(torch.round(big / torch.exp2(e)) > most, e + 1, e)
    q = torch.round(v / torch.exp2(e))
    return torch.where((q < 1) & (v > 0) & (most == 255), 1.0, q) * torch.exp2(e)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "pack":
        most = 255 if case["rectified"] else 127
        return torch.cat([torch.cat([_held_of(v, most) for v in x.split(BLOCK, 1)], 1) for x in s["x"].split(1 << 16)])
    if op == "int8":
        w, out = s["w"].double() * s["ws"].double()[:, None], []
        for x in s["x"].split(1 << 16):
            x = x.double()
            step = torch.clamp(torch.amax(torch.abs(x), 1, keepdim=True) / 127, min=2.0 ** -126).float().double()
            out.append(torch.addmm(s["b"].double(), torch.round(x / step) * step, w.t()))
        y = torch.cat(out)
        return torch.clamp(y, min=0) if case["relu"] else y
    n, starts = case["n"], [0]
    for size in s.get("sizes", [n]):
        starts.append(starts[-1] + size)
    weights = s["w"].double() if "sizes" in s else s["w"].double()[None]
    ys, gxs, gws, gbs = [], [], [], []
    for g, w in enumerate(weights):
        gw = torch.zeros_like(w)
        gb = torch.zeros(case["d_out"], device=DEV, dtype=torch.float64)
        for a in range(starts[g], starts[g + 1], 1 << 16):
            at = slice(a, min(a + (1 << 16), starts[g + 1]))
            x = _held(s["codes"][at], s["exponents"][at]) if op == "packed_grad" else s["x"][at].double()
            if op == "grouped":
                y = torch.addmm(s["b"][g].double(), x, w.t())
                ys.append(torch.clamp(y, min=0) if case["relu"] else y)
                continue
            gz = s["gz"][at].double()
            gw += torch.mm(gz.t(), x)
            gb += gz.sum(0)
            if case["want_x"]:
                back = torch.mm(gz, w)
                gxs.append(torch.where(x > 0, back, 0.0) if case.get("relu", case.get("rectified")) else back)
        gws.append(gw)
        gbs.append(gb)
    if op == "grouped":
        return torch.cat(ys)
    gx = torch.cat(gxs) if case["want_x"] else None
    if op == "packed_grad":
        return gx, gws[0], gbs[0]
    return gx, torch.stack(gws), torch.stack(gbs)
