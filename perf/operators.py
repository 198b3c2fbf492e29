"""Cases of the operators around the low-rank path: the step of the parameters that are kept dense (AdamW over many
tensors, states in 32 or 8 bits), the global norm of the gradients before it, and the 8-bit product of the linear layers
with a scale for each block of 128, with the quantiser that makes its operands.

`run` computes an operator in plain torch operations, or, where `own` is true, by the library's calls.  What the library
holds in 8 bits is a torch float8 tensor on both sides (its values times powers of two that are returned beside it)."""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

# hidden width, intermediate width, layers of the models whose blocks the benchmark runs
MODELS = {"60m": (512, 1376, 8), "130m": (768, 2048, 12), "350m": (1024, 2736, 24), "1b": (2048, 5461, 24)}
VOCAB = 32000
BLOCK = 256                     # elements that share a scale of an 8-bit state
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4, "e5m2": E5}
SIZE = {"f32": 4, "bf16": 2}
MASK = 0xFFFFFFFF


# ------------------------------------------------------------------ cases
def listed():
    return [
        # the gains of the norms of the smallest model: what is left dense when every matrix is low-rank; latency
        dict(name="adamw gains 60m", op="adamw", part="gains", model="60m", layers=8, p="f32", g="f32", state=32, copy=False, gap=256, t=7),
        # the dense baseline: every block of a model, fp32 masters, bf16 gradients and a bf16 copy for the next forward pass
        dict(name="adamw blocks 130m", op="adamw", part="blocks", model="130m", layers=12, p="f32", g="bf16", state=32, copy=True, gap=256, t=1000),
        # ragged tensors packed one behind the other in flat buffers: nothing is aligned
        dict(name="adamw packed ragged", op="adamw", part="mixed", sizes=5, tensors=60, most=1 << 21, p="f32", g="f32", state=32, copy=False, gap=1, t=1),
        # embedding and output head of the largest model, dense, 8-bit states
        dict(name="adamw8 tables 1b", op="adamw", part="tables", model="1b", layers=2, p="f32", g="bf16", state=8, copy=False, gap=256, t=200),
        # bf16 parameters without masters, 8-bit states: the least memory
        dict(name="adamw8 blocks 350m bf16", op="adamw", part="blocks", model="350m", layers=8, p="bf16", g="bf16", state=8, copy=False, gap=256, t=3),
        # the norm before a step: small and large
        dict(name="norm gains 60m", op="norm", part="gains", model="60m", layers=8, g="f32", gap=256),
        dict(name="norm blocks 1b", op="norm", part="blocks", model="1b", layers=6, g="bf16", gap=256),
        # a weight for the forward and the backward product; the gradient of a layer's output for both of its products
        dict(name="quantize weight 1b", op="quantize", m=2048, n=5461, x="f32", q="e4m3", rows=128, plain=True, turned=True),
        dict(name="quantize gradient", op="quantize", m=16384, n=2048, x="bf16", q="e5m2", rows=1, plain=True, turned=True),
        # one token; the weight gradient of a ragged batch; the output head over a batch.  The result is bf16: a matrix
        # instruction aligns the products of eight neighbours to the largest and keeps 14 bits, which 32 bits would not show
        dict(name="matmul token", op="matmul", m=1, n=5461, k=2048, a="e4m3", b="e4m3", a_rows=1, b_rows=128),
        dict(name="matmul weight gradient", op="matmul", m=2736, n=1024, k=12345, a="e5m2", b="e4m3", a_rows=1, b_rows=1),
        dict(name="matmul head", op="matmul", m=8192, n=VOCAB, k=2048, a="e4m3", b="e4m3", a_rows=1, b_rows=128),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["adamw", "adamw", "norm", "quantize", "matmul", "matmul"])
    if op in ("adamw", "norm"):
        c = dict(op=op, part="mixed", sizes=rng.randrange(1 << 30), tensors=_log(rng, 1, 200), most=_log(rng, 64, 1 << 21), g=rng.choice(["f32", "bf16"]))
        c["gap"] = 256
        if op == "adamw":
            c |= dict(p=rng.choice(["f32", "bf16"]), state=rng.choice([32, 8]), t=_log(rng, 1, 100000))
            c["copy"] = c["p"] == "f32" and rng.random() < 0.5
            if c["p"] == "f32" and c["state"] == 32:
                c["gap"] = rng.choice([1, 256])
        return c
    if op == "quantize":
        both = rng.choice([(True, False), (True, True), (False, True)])
        return dict(op=op, m=_log(rng, 1, 16384), n=_log(rng, 1, 8192), x=rng.choice(["f32", "bf16"]), q=rng.choice(["e4m3", "e5m2"]), rows=rng.choice([1, 128]),
                    plain=both[0], turned=both[1])
    m, n, k = _log(rng, 1, 16384), _log(rng, 16, 8192), _log(rng, 64, 8192)
    return dict(op=op, m=m, n=n, k=k, a=rng.choice(["e4m3", "e5m2"]), b="e4m3", a_rows=1, b_rows=rng.choice([1, 128]))


def _sizes(case):
    """(counts of the tensors with weight decay, counts of those without)"""
    if case["part"] == "mixed":
        rng = random.Random(case["sizes"])
        n = [_log(rng, 1, case["most"]) for _ in range(case["tensors"])]
        return n[: len(n) // 2], n[len(n) // 2:]
    h, f, _ = MODELS[case["model"]]
    if case["part"] == "tables":
        return [VOCAB * h] * case["layers"], []
    gains = [h] * (2 * case["layers"] + 1)
    return ([h * h] * 4 + [h * f] * 3) * case["layers"] if case["part"] == "blocks" else [], gains


def _blocks(m, n, rows):
    return -(-m // rows) * -(-n // 128)


def work(case):
    if case["op"] in ("adamw", "norm"):
        n = sum(sum(s) for s in _sizes(case))
        if case["op"] == "norm":
            return {"bytes": n * SIZE[case["g"]] + 8, "flops": 2 * n}
        state = 16 if case["state"] == 32 else 4 + 4 / BLOCK
        return {"bytes": n * (2 * SIZE[case["p"]] + SIZE[case["g"]] + state + (2 if case["copy"] else 0)), "flops": 20 * n}
    m, n = case["m"], case["n"]
    if case["op"] == "quantize":
        r = case["rows"]
        out = (m * n + _blocks(m, n, r)) * case["plain"] + (m * n + _blocks(n, m, r)) * case["turned"]
        return {"bytes": m * n * SIZE[case["x"]] + out, "flops": 3 * m * n}
    k = case["k"]
    return {"bytes": m * k + n * k + _blocks(m, k, case["a_rows"]) + _blocks(n, k, case["b_rows"]) + m * n * 2, "flops": 2 * m * n * k}


# ------------------------------------------------------------------ numbers that both forms are defined by
def _mix(h):
    """A 32-bit mix of an integer, or of an int64 tensor of values below 2^32."""
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & MASK
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & MASK
    return h ^ (h >> 16)


def _key(seed, t, j):
    """The key of the j-th tensor's random bits in step t."""
    return _mix((_mix(_mix(_mix(seed & MASK) ^ (seed >> 32)) ^ t) + j * 0x9E3779B1) & MASK)


def _two_to(b):
    """2^(b - 127) as fp32 for scale bytes 1 .. 254."""
    return (b.int() << 23).view(torch.float32)


def _f(x):
    return float(np.float32(x))


# ------------------------------------------------------------------ inputs
def _randn(n, gen, scale=1.0):
    return torch.randn(n, generator=gen, device="cuda") * scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "quantize":
        m, n = case["m"], case["n"]
        x = torch.randn(m, n, generator=gen, device="cuda")
        x *= torch.exp(torch.randn(n, generator=gen, device="cuda"))            # channels of different size
        s["x"] = (x * 1e-2).to(DTYPES[case["x"]])
        s["q"] = _empty(m, n, case["q"], case["rows"]) if case["plain"] else (None, None)
        s["qt"] = _empty(n, m, case["q"], case["rows"]) if case["turned"] else (None, None)
        return s
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        for name, rows, dt, size in (("a", m, case["a"], 1.0), ("b", n, case["b"], 0.02)):
            x = torch.randn(rows, k, generator=gen, device="cuda") * size
            x *= torch.exp(0.5 * torch.randn(k, generator=gen, device="cuda"))
            q, b = _quantize(x, case[name + "_rows"], DTYPES[dt])
            s[name] = _empty(rows, k, dt, case[name + "_rows"])
            s[name][0].copy_(q)
            s[name][1].copy_(b)
            del x, q
        s["c"] = torch.zeros(m, n, device="cuda", dtype=torch.bfloat16)
        if own:
            import paper_2602_08007_amd as tsr
            nbytes = tsr.tsr_fp8_matmul_workspace_bytes(m, n, k)
            s["ws"] = tsr.workspace(nbytes) if nbytes else None
        return s
    decayed, rest = _sizes(case)
    gap, places, at = case["gap"], [], 0
    for n in decayed + rest:
        places.append((at, n))
        at += -(-n // gap) * gap
    total = -(-at // BLOCK) * BLOCK
    live = torch.zeros(total, dtype=torch.bool, device="cuda")
    ends = torch.zeros(total + 1, dtype=torch.int32, device="cuda")
    ends.index_add_(0, torch.tensor([a for a, n in places], device="cuda"), torch.ones(len(places), dtype=torch.int32, device="cuda"))
    ends.index_add_(0, torch.tensor([a + n for a, n in places], device="cuda"), -torch.ones(len(places), dtype=torch.int32, device="cuda"))
    live = ends[:-1].cumsum(0) > 0
    del ends
    # gradients of different size from stretch to stretch, as tensors and rows have them
    size = torch.exp(_randn(total // BLOCK, gen)).repeat_interleave(BLOCK) * 1e-3 * live
    s["g"] = (_randn(total, gen) * size).to(DTYPES[case["g"]])
    if case["op"] == "norm":
        s["norm"], s["coef"] = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        if own:
            import paper_2602_08007_amd as tsr
            s["set"] = tsr.TensorSet([dict(g=s["g"][a:a + n]) for a, n in places])
            s["ws"] = tsr.workspace(tsr.tsr_grad_norm_workspace_bytes(s["set"]))
        return s
    p = _randn(total, gen, 0.02) * live
    s["p"] = p.to(DTYPES[case["p"]])
    if case["copy"]:
        s["p16"] = p.bfloat16()
    del p
    m = _randn(total, gen, 0.3) * size
    v = (size * torch.exp(0.5 * _randn(total, gen))).square()
    del size, live
    if case["state"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["ms"] = (x.reshape(-1) for x in _quantize(m.view(-1, BLOCK), 1, E4, BLOCK))
        s["v"], s["vs"] = (x.reshape(-1) for x in _quantize(v.view(-1, BLOCK), 1, E5, BLOCK))
    del m, v
    s["coef"] = torch.full((1,), 0.37, device="cuda")
    s["seed"] = 1 + seed * 0x1234567 % (1 << 60)
    s["split"] = sum(-(-n // gap) * gap for n in decayed)          # where the tensors without weight decay begin
    if case["state"] == 8 or case["p"] == "bf16":
        # for the plain form: the key of each block's tensor, and the block's first index in its tensor
        reps = torch.tensor([-(-n // BLOCK) for a, n in places], device="cuda")
        first = torch.tensor([a // BLOCK for a, n in places], device="cuda")
        keys = torch.tensor([_key(s["seed"], case["t"], j) for j in range(len(places))], device="cuda")
        s["keys"] = keys.repeat_interleave(reps)
        s["base"] = (torch.arange(total // BLOCK, device="cuda") - first.repeat_interleave(reps)) * BLOCK
    if own:
        import paper_2602_08007_amd as tsr
        tensors = []
        for i, (a, n) in enumerate(places):
            d = dict(p=s["p"][a:a + n], g=s["g"][a:a + n], m=s["m"][a:a + n], v=s["v"][a:a + n], wd_scale=1.0 if i < len(decayed) else 0.0)
            if case["state"] == 8:
                d |= dict(m_scale=s["ms"][a // BLOCK:(a + n + BLOCK - 1) // BLOCK], v_scale=s["vs"][a // BLOCK:(a + n + BLOCK - 1) // BLOCK])
            if case["copy"]:
                d["p16"] = s["p16"][a:a + n]
            tensors.append(d)
        s["set"] = tsr.TensorSet(tensors)
    return s


def _empty(m, n, q, rows):
    """Place for an 8-bit matrix and its scale bytes, rows padded to 16 bytes and to 4 scales."""
    x = torch.zeros(m, -(-n // 16) * 16, device="cuda", dtype=torch.uint8).view(DTYPES[q])[:, :n]
    return x, torch.zeros(-(-m // rows), -(-n // 512) * 4, device="cuda", dtype=torch.uint8)[:, : -(-n // 128)]


# ------------------------------------------------------------------ plain forms
LR, WD, B1, B2, EPS, SCALE = 1e-3, 0.1, 0.9, 0.999, 1e-8, 1.0
MAX_NORM = 1.0


def _scale_bytes(amax, q):
    """The least power of two that brings amax to 448 (e4m3) or 57344 (e5m2) at most, as an exponent byte; 127 for nothing."""
    f, x = torch.frexp(amax)                                       # amax = f 2^x, 1/2 <= f < 1
    e = x - (9 if q == E4 else 16) + (f > 0.875).int()
    return torch.where(amax > 0, (e + 127).clamp(1, 254), 127)


def _finite_max(x, dim):
    x = x.abs()
    return torch.where(torch.isfinite(x), x, 0.0).amax(dim)


def _quantize(x, rows, q, cols=128):
    """x (fp32) in blocks of rows x cols: nearest values of type q, and the exponent bytes."""
    m, n = x.shape
    mb, nb = -(-m // rows), -(-n // cols)
    full = torch.nn.functional.pad(x, (0, nb * cols - n, 0, mb * rows - m)).view(mb, rows, nb, cols)
    b = _scale_bytes(_finite_max(full, (1, 3)), q)
    y = full * _two_to(254 - b)[:, None, :, None]
    return y.view(mb * rows, nb * cols)[:m, :n].to(q), b.to(torch.uint8)


def _random_bits(s):
    """32 bits for each element, from its index in its tensor and the tensor's key."""
    i = (s["base"][:, None] + torch.arange(BLOCK, device="cuda")).reshape(-1)
    return _mix(((i & MASK) * 0x9E3779B1 + s["keys"].repeat_interleave(BLOCK) + (i >> 32) * 0x7FEB352D) & MASK)


def _state8(x, q, r, bits):
    """x in blocks of BLOCK as type q, rounded up with the probability of what it is above the value below (r: 16 bits)."""
    b = _scale_bytes(_finite_max(x.view(-1, BLOCK), 1), q)
    y = (x.view(-1, BLOCK) * _two_to(254 - b)[:, None]).reshape(-1)
    a = y.abs()
    drop, least, low, inf = (20, 2.0 ** -6, 512.0, 0x7F) if q == E4 else (21, 2.0 ** -14, 65536.0, 0x7C)
    r = r.int()
    code = ((a.view(torch.int32) + (r << (drop - 16))) >> drop) - ((120 << 3) if q == E4 else (112 << 2))
    code = torch.where(a < least, torch.floor(a * low + r * 2.0 ** -16).int(), code)
    if q == E5:
        code = torch.where((a > 0) & (code < 1), 1, code)          # a positive second moment stays positive
    code = torch.where(torch.isinf(a), inf, torch.where(torch.isnan(a), 0x7F, code)) | torch.where(torch.signbit(y), 0x80, 0)
    return code.to(torch.uint8).view(q), b.to(torch.uint8)


def _plain_adamw(s):
    case = s["case"]
    lr, wd, b1, b2, eps = (_f(x) for x in (LR, WD, B1, B2, EPS))
    c1, c2 = _f(1 / (1 - b1 ** case["t"])), _f(1 / (1 - b2 ** case["t"]))
    g = s["g"].float() * s["coef"]
    m, v = s["m"].float(), s["v"].float()
    if case["state"] == 8:
        m, v = ((x.view(-1, BLOCK) * _two_to(b)[:, None]).reshape(-1) for x, b in ((m, s["ms"]), (v, s["vs"])))
    m = m * b1 + g * _f(np.float32(1) - np.float32(b1))
    v = v * b2 + (g * g) * _f(np.float32(1) - np.float32(b2))
    del g
    d = (m * c1) / (torch.sqrt(v * c2) + eps)
    p = s["p"].float()
    p[: s["split"]] *= _f(1 - lr * wd)
    p -= d * _f(lr * SCALE)
    del d
    h = _random_bits(s) if "keys" in s else None
    if case["state"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["ms"] = _state8(m, E4, h & 0xFFFF, 4)
        s["v"], s["vs"] = _state8(v, E5, h >> 16, 5)
    if case["p"] == "f32":
        s["p"] = p
    else:
        r = ((h * 0x9E3779B1) & MASK) >> 16
        up = ((p.view(torch.int32) + r.int()) & -65536).view(torch.float32)
        s["p"] = torch.where(torch.isfinite(p), up, p).bfloat16()
    if case["copy"]:
        s["p16"] = p.bfloat16()


def _wide(x, rows, m, n):
    """Scale bytes of blocks of rows x 128 as fp32 factors of the elements."""
    x = _two_to(x).repeat_interleave(128, 1)[:, :n]
    return x.repeat_interleave(rows, 0)[:m] if rows > 1 else x


def run(s):
    case = s["case"]
    if own:
        import paper_2602_08007_amd as tsr
    if case["op"] == "adamw":
        if own:
            tsr.tsr_adamw_batched(s["set"], case["t"], LR, wd=WD, beta1=B1, beta2=B2, eps=EPS, scale=SCALE, g_scale=s["coef"], seed=s["seed"])
        else:
            _plain_adamw(s)
        return {k: s[k] for k in ("p", "m", "v", "ms", "vs", "p16") if k in s}
    if case["op"] == "norm":
        if own:
            tsr.tsr_grad_norm_batched(s["set"], MAX_NORM, s["norm"], s["coef"], ws=s["ws"])
            return {"norm": s["norm"], "coef": s["coef"]}
        norm = s["g"].double().square().sum().sqrt()
        coef = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
        return {"norm": norm.float().view(1), "coef": torch.where(torch.isfinite(norm), coef, math.nan).float().view(1)}
    if case["op"] == "quantize":
        if own:
            tsr.tsr_fp8_quantize(s["x"], *s["q"], *s["qt"], block_rows=case["rows"])
            return {"q": s["q"], "qt": s["qt"]}
        x = s["x"].float()
        q = _quantize(x, case["rows"], DTYPES[case["q"]]) if case["plain"] else (None, None)
        qt = _quantize(x.t(), case["rows"], DTYPES[case["q"]]) if case["turned"] else (None, None)
        return {"q": q, "qt": qt}
    if own:
        tsr.tsr_fp8_matmul(*s["a"], *s["b"], s["c"], ws=s["ws"])
        return s["c"]
    m, n, k = case["m"], case["n"], case["k"]
    a, b = s["a"][0].float() * _wide(s["a"][1], case["a_rows"], m, k), s["b"][0].float() * _wide(s["b"][1], case["b_rows"], n, k)
    s["c"] = torch.matmul(a, b.t()).bfloat16()
    return s["c"]


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_state(x, top, mant, least, r):
    """x (fp64) in blocks of BLOCK on the values f 2^e with `mant` fraction bits, times a power of two for each block."""
    y = x.view(-1, BLOCK)
    amax = y.abs().amax(1, keepdim=True)
    e = torch.ceil(torch.log2(amax.clamp_min(1e-300) / top))
    e = torch.where(amax > 0, e, 0.0).clamp(-126, 127)
    y = (y / torch.exp2(e)).reshape(-1)
    octave = torch.floor(torch.log2(y.abs().clamp_min(1e-300)))
    octave = octave + (torch.exp2(octave + 1) <= y.abs()).double() - (torch.exp2(octave) > y.abs()).double()
    step = torch.exp2(octave.clamp_min(least) - mant)
    low = torch.floor(y.abs() / step + r / 65536.0)
    if least == -14:
        low = torch.where(y > 0, low.clamp_min(1.0), low)
    return torch.sign(y) * low * step


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "norm":
        parts = [x.double() @ x.double() for x in s["g"].split(1 << 24)]
        norm = math.sqrt(math.fsum(float(x) for x in parts))
        return {"norm": torch.tensor([norm], dtype=torch.float64), "coef": torch.tensor([min(1.0, MAX_NORM / norm) if norm else 1.0], dtype=torch.float64)}
    if case["op"] == "quantize":
        out = {}
        for name, x, wanted in (("q", s["x"].double(), case["plain"]), ("qt", s["x"].double().t(), case["turned"])):
            if not wanted:
                out[name] = (None, None)
                continue
            rows, top, mant, least = case["rows"], *((448.0, 3, -6) if case["q"] == "e4m3" else (57344.0, 2, -14))
            y = torch.empty_like(x)
            size = torch.nn.functional.max_pool2d(x.abs()[None, None], (rows, 128), ceil_mode=True)[0, 0]
            e = torch.where(size > 0, torch.ceil(torch.log2(size.clamp_min(1e-300) / top)), 0.0)
            y = x / torch.exp2(e).repeat_interleave(rows, 0)[: x.shape[0]].repeat_interleave(128, 1)[:, : x.shape[1]]
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(1e-300))).clamp_min(least) - mant)
            out[name] = (torch.round(y / step) * step, None)
        return out
    if case["op"] == "matmul":
        a, b = (s[x][0].double() * torch.exp2(s[x][1].double() - 127).repeat_interleave(case[x + "_rows"], 0)[: s[x][0].shape[0]].repeat_interleave(128, 1)[:, : case["k"]]
                for x in ("a", "b"))
        return torch.matmul(a, b.t())
    b1, b2 = _f(B1), _f(B2)
    g = s["g"].double() * s["coef"].double()
    m, v = s["m"].double(), s["v"].double()
    if case["state"] == 8:
        m = m * torch.exp2(s["ms"].double() - 127).repeat_interleave(BLOCK)
        v = v * torch.exp2(s["vs"].double() - 127).repeat_interleave(BLOCK)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    d = (m / (1 - b1 ** case["t"])) / (torch.sqrt(v / (1 - b2 ** case["t"])) + _f(EPS))
    p = s["p"].double()
    decay = torch.where(torch.arange(p.numel(), device="cuda") < s["split"], _f(WD), 0.0).double()
    p = p - _f(LR) * (SCALE * d + decay * p)
    del d, decay, g
    out = {"p16": p} if case["copy"] else {}
    if "keys" in s:
        i = torch.arange(BLOCK, device="cuda") + s["base"][:, None]
        h = _mix((i % (1 << 32) * 0x9E3779B1 + s["keys"][:, None] + i // (1 << 32) * 0x7FEB352D) % (1 << 32)).reshape(-1)
    if case["p"] == "bf16":
        step = torch.exp2(torch.floor(torch.log2(p.abs().clamp_min(1e-300))) - 7)
        p = torch.sign(p) * torch.floor(p.abs() / step + (h * 0x9E3779B1 % (1 << 32) // 65536) / 65536.0) * step
    out["p"] = p
    if case["state"] == 32:
        return out | {"m": m, "v": v}
    return out | {"m": _exact_state(m, 448.0, 3, -6, h % 65536), "v": _exact_state(v, 57344.0, 2, -14, h // 65536), "ms": None, "vs": None}
