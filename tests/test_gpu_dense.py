"""AdamW over many tensors and the norm of many gradients, against the formulas in fp64.

Bounds are counted in roundings: u = 2^-24 is half a step of fp32 relative to the value, 2^-8 of bf16.  8-bit moments and bf16
parameters are rounded stochastically by a hash that is computed here too; a stored value may differ from the one that the
fp64 formula gives only where that formula is within its fp32 error of the border between two values."""
import numpy as np
import pytest
import torch

import synth_inputs as si

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
HYPER = dict(lr=1e-2, wd=0.1, beta1=0.9, beta2=0.999, eps=1e-8, scale=0.5)


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_amd as t
    assert torch.cuda.is_available()
    return t


def f32(x):
    return float(np.float32(x))


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def draw(n, *key, std=1.0):
    return si.normal((n,), si.stream_key(*key)).mul_(std)


def offset(x, shift):
    """x on the GPU, `shift` elements into a buffer whose other elements are a pattern; (view, check that the pattern is whole)."""
    size = x.element_size()
    buf = torch.full(((x.numel() + shift + 64) * size,), 0xA5, dtype=torch.uint8, device="cuda")
    body = slice(shift * size, (shift + x.numel()) * size)
    view = buf[body].view(x.dtype)
    view.copy_(x.to("cuda"))
    def whole():
        rest = buf.clone()
        rest[body] = 0xA5
        return bool((rest == 0xA5).all())
    return view, whole


# ------------------------------------------------------------------ formulas
def mix(h):
    h = np.asarray(h, dtype=np.uint32)
    with np.errstate(over="ignore"):
        h = (h ^ (h >> np.uint32(16))) * np.uint32(0x85EBCA6B)
        h = (h ^ (h >> np.uint32(13))) * np.uint32(0xC2B2AE35)
    return h ^ (h >> np.uint32(16))


def hash_bits(seed, t, j, n):
    with np.errstate(over="ignore"):
        key = mix(mix(mix(np.uint32(seed & 0xFFFFFFFF)) ^ np.uint32(seed >> 32)) ^ np.uint32(t))
        key = mix(key + np.uint32(j * 0x9E3779B1 & 0xFFFFFFFF))
        return mix(np.arange(n, dtype=np.uint32) * np.uint32(0x9E3779B1) + key)


def step64(p, g, m, v, t, h, gs=1.0, wd_scale=1.0, ratio=7):
    """(p, m, v, bounds of their fp32 errors) of one step in fp64.  ratio: roundings of the quotient, in half steps: constants 1.5,
    products 1.5, root 1, sum 1, quotient 1 make 6 (7 with what is left); beside 8-bit states root and reciprocal may be off by a
    whole step of fp32 (2 each) and their product is rounded once more: 1.5 + 1.5 + 2 + 1 + 2 + 1 = 9 (10)."""
    b1, b2 = f32(h["beta1"]), f32(h["beta2"])
    o1, o2 = f32(np.float32(1) - np.float32(b1)), f32(np.float32(1) - np.float32(b2))
    lr, wd, eps, scale = f32(h["lr"]), f32(h["wd"]), f32(h["eps"]), f32(h["scale"])
    g = g * gs
    m2, v2 = b1 * m + o1 * g, b2 * v + o2 * g * g
    em = U * (2 * b1 * np.abs(m) + 3 * o1 * np.abs(g)) * 1.01 + 1e-44         # products and the sum; g was scaled
    ev = U * (2 * b2 * v + 5 * o2 * g * g) * 1.01 + 1e-44
    c1, c2 = 1 / (1 - b1 ** t), 1 / (1 - b2 ** t)
    den = np.sqrt(v2 * c2) + eps
    d = m2 * c1 / den
    rv = np.divide(ev, v2, out=np.zeros_like(ev), where=v2 > 0)
    ed = em * c1 / den + np.abs(d) * (0.5 * rv + ratio * U)
    decay, step = 1 - lr * wd * wd_scale, lr * scale
    out = decay * p - step * d
    ep = (step * ed + U * (3 * np.abs(decay * p) + 4 * step * np.abs(d))) * 1.01 + 1e-44
    return out, m2, v2, ep, em, ev


def state_rule(y, ey, r16, mant, least, positive):
    """(value by the rule, whether the rule is sure of it) for y >= 0 on a grid of `mant` fraction bits from 2^least down."""
    octave = np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), least)
    step = 2.0 ** (octave - mant)
    place = y / step + r16 / 65536.0
    low = np.floor(place)
    err = ey / step + 2.0 ** -20                                              # and the sum's rounding below the least octave
    sure = (np.abs(place - np.rint(place)) > err) & (np.abs(y / 2.0 ** np.rint(np.log2(np.maximum(y, 1e-300))) - 1) > 1e-6)
    if positive:
        low = np.where(y > 0, np.maximum(low, 1), low)
    return low * step, sure


def check_state(q, b, x, ex, r16, fmt):
    """8-bit values q and scale bytes b against x (fp64) with error bounds ex."""
    n = x.size
    top, mant, least = (448.0, 3, -6) if fmt == E4 else (57344.0, 2, -14)
    pad = -n % 256
    big = np.pad(np.abs(x), (0, pad)).reshape(-1, 256).max(1)
    at = np.pad(np.abs(x), (0, pad)).reshape(-1, 256).argmax(1)
    e = np.where(big > 0, np.ceil(np.log2(np.maximum(big, 1e-300) / top)), 0).clip(-126, 127)
    border = np.abs(np.log2(np.maximum(big, 1e-300) / top) - np.rint(np.log2(np.maximum(big, 1e-300) / top))) < 1e-5
    got = b.cpu().numpy().astype(int)
    assert np.all((got == e + 127) | border), "scale bytes"
    scale = (2.0 ** (got - 127.0)).repeat(256)[:n]
    values = f64(q)
    y = np.abs(x) / scale
    want, sure = state_rule(y, ex / scale, r16, mant, least, fmt == E5)
    step = np.maximum(2.0 ** (np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), least) - mant), 1e-300)
    assert np.all(np.abs(np.abs(values) - y) <= step * (1 + 1e-4) + ex / scale), "not a neighbour"
    assert np.all(np.abs(values[sure]) == want[sure]), "not the neighbour that the bits choose"
    assert sure.mean() > 0.9 or n < 100
    live = np.abs(values) > 0
    assert np.all((values[live] < 0) == (x[live] < 0))


# ------------------------------------------------------------------ 32-bit states
@pytest.mark.parametrize("pt,gt", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("n,shift", [(1, 0), (3, 1), (255, 0), (4096, 0), (4097, 3), (70001, 0), (70001, 1)])
def test_adamw_states_in_32_bits(tsr, pt, gt, n, shift):
    t, seed = 5, 0x1234567890
    p, wp = offset(draw(n, 1, n).to(pt), shift)
    g, wg = offset(draw(n, 2, n, std=0.1).to(gt), shift)
    m, wm = offset(draw(n, 3, n, std=0.1), shift)
    v, wv = offset(draw(n, 4, n, std=0.1).square(), shift)
    p16, wc = offset(torch.zeros(n, dtype=torch.bfloat16), shift)
    tensor = dict(p=p, g=g, m=m, v=v, wd_scale=0.5)
    if pt == torch.float32:
        tensor["p16"] = p16
    want, m2, v2, ep, em, ev = step64(f64(p), f64(g), f64(m), f64(v), t, HYPER, wd_scale=0.5)
    tsr.tsr_adamw_batched([tensor], t, seed=seed, **HYPER)
    torch.cuda.synchronize()
    assert np.all(np.abs(f64(m) - m2) <= em) and np.all(np.abs(f64(v) - v2) <= ev)
    got = f64(p)
    if pt == torch.float32:
        assert np.all(np.abs(got - want) <= ep)
        assert torch.equal(p16, p.bfloat16())
    else:
        with np.errstate(over="ignore"):
            r = (hash_bits(seed, t, 0, n) * np.uint32(0x9E3779B1)) >> np.uint32(16)
        value, sure = state_rule(np.abs(want), ep, r, 7, -126, False)
        assert np.all(np.abs(got - want) <= 2.0 ** -7 * np.abs(want) * (1 + 1e-4) + ep)
        assert np.all(np.abs(got[sure]) == value[sure])
    assert wp() and wg() and wm() and wv() and (wc() if pt == torch.float32 else True)


def test_many_tensors_empty_ones_among_them(tsr):
    sizes = [0, 1, 513, 4096, 0, 5000] * 20 + [9]                             # more than three launches hold
    rows = []
    for j, n in enumerate(sizes):
        rows.append(dict(p=draw(n, 5, j).cuda(), g=draw(n, 6, j, std=1e-2).cuda(), m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"),
                         wd_scale=float(j % 2)))
    want = [step64(f64(r["p"]), f64(r["g"]), f64(r["m"]), f64(r["v"]), 1, HYPER, gs=f32(0.25), wd_scale=r["wd_scale"]) for r in rows]
    tsr.tsr_adamw_batched(rows, 1, g_scale=torch.tensor([0.25], device="cuda"), **HYPER)
    torch.cuda.synchronize()
    for r, w in zip(rows, want):
        assert np.all(np.abs(f64(r["p"]) - w[0]) <= w[3]) and np.all(np.abs(f64(r["m"]) - w[1]) <= w[4]) and np.all(np.abs(f64(r["v"]) - w[2]) <= w[5])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_step_whose_factor_is_not_finite_is_left_out(tsr, value):
    n = 3000
    row = dict(p=draw(n, 7).cuda(), g=draw(n, 8).cuda(), m=draw(n, 9).cuda(), v=draw(n, 10).square().cuda())
    row8 = eight(n, 11)
    before = [x.clone() for r in (row, row8) for x in r.values() if isinstance(x, torch.Tensor)]
    tsr.tsr_adamw_batched([row, row8], 2, 1e-2, g_scale=torch.tensor([value], device="cuda"))
    torch.cuda.synchronize()
    after = [x for r in (row, row8) for x in r.values() if isinstance(x, torch.Tensor)]
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, after))


def test_gradients_that_are_not_finite_spoil_their_own_element_only(tsr):
    n, t = 1000, 4
    g = draw(n, 12, std=1e-2)
    bad = [0, 255, 256, 700, 999]
    g[bad[0]], g[bad[1]], g[bad[2]], g[bad[3]], g[bad[4]] = float("nan"), float("inf"), -float("inf"), float("nan"), float("inf")
    for row in (dict(p=draw(n, 13).cuda(), g=g.cuda(), m=draw(n, 14, std=1e-2).cuda(), v=draw(n, 15, std=1e-2).square().cuda()), dict(eight(n, 16), g=g.cuda())):
        clean = {k: x.clone() if isinstance(x, torch.Tensor) else x for k, x in row.items()}
        clean["g"][bad] = 0
        tsr.tsr_adamw_batched([row], t, **HYPER)
        tsr.tsr_adamw_batched([clean], t, **HYPER)
        torch.cuda.synchronize()
        keep = torch.ones(n, dtype=torch.bool)
        keep[bad] = False
        for k in ("p", "m", "v"):
            a, b = row[k].float().cpu(), clean[k].float().cpu()
            assert not torch.isfinite(a[bad]).any(), k
            # without the element's own value the scale of its block may be another: values, not codes, are compared
            if row[k].dtype in (E4, E5):
                s = "m_scale" if k == "m" else "v_scale"
                a, b = (x * torch.exp2(r[s].cpu().float() - 127).repeat_interleave(256)[:n] for x, r in ((a, row), (b, clean)))
                assert torch.allclose(a[keep], b[keep], rtol=0.26, atol=0)
            else:
                assert torch.equal(a[keep], b[keep]), k


# ------------------------------------------------------------------ 8-bit states
def eight(n, key, pt=torch.float32, gt=torch.float32, shift=0):
    """A tensor with 8-bit states that hold something."""
    blocks = -(-n // 256)
    size = torch.exp(draw(blocks, key, 5)).repeat_interleave(256)[:n] * 1e-2
    m8 = (draw(n, key, 1) * 50).to(E4)
    v8 = (draw(n, key, 2).square() * 1000 + 2.0 ** -14).to(E5)
    row = dict(p=draw(n, key, 3).to(pt), g=(draw(n, key, 4) * size).to(gt), m=m8, v=v8)
    row = {k: offset(x, shift)[0] for k, x in row.items()}
    row["m_scale"] = (torch.full((blocks,), 112) + (torch.arange(blocks) % 3)).to(torch.uint8).cuda()
    row["v_scale"] = (torch.full((blocks,), 97) + (torch.arange(blocks) % 5)).to(torch.uint8).cuda()
    return row


def value_of(row, name, n):
    return f64(row[name]) * (2.0 ** (row[name + "_scale"].cpu().numpy().astype(float) - 127)).repeat(256)[:n]


@pytest.mark.parametrize("pt,gt", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("n,shift", [(1, 0), (256, 0), (257, 0), (5000, 0), (70001, 0), (70001, 1)])
def test_adamw_states_in_8_bits(tsr, pt, gt, n, shift):
    t, seed = 37, 99
    row = eight(n, 20, pt, gt, shift)
    m, v = value_of(row, "m", n), value_of(row, "v", n)
    want, m2, v2, ep, em, ev = step64(f64(row["p"]), f64(row["g"]), m, v, t, HYPER, ratio=10)
    first = dict(p=torch.zeros(1, device="cuda"), g=torch.zeros(1, device="cuda"), m=torch.zeros(1, device="cuda"), v=torch.zeros(1, device="cuda"))
    tsr.tsr_adamw_batched([first, row], t, seed=seed, **HYPER)
    torch.cuda.synchronize()
    h = hash_bits(seed, t, 1, n)
    check_state(row["m"], row["m_scale"], m2, em, (h & 0xFFFF).astype(np.float64), E4)
    check_state(row["v"], row["v_scale"], v2, ev, (h >> 16).astype(np.float64), E5)
    got = f64(row["p"])
    if pt == torch.float32:
        assert np.all(np.abs(got - want) <= ep)
    else:
        assert np.all(np.abs(got - want) <= 2.0 ** -7 * np.abs(want) * (1 + 1e-4) + ep)


def test_8_bit_states_from_zero_and_a_second_moment_that_stays_positive(tsr):
    n = 2048
    g = draw(n, 30) * 1e-3
    g[1::2] *= 1e-9                                                           # squares 2^-60 of the block's largest: below the type's least
    g[4] = 0
    row = dict(p=torch.zeros(n), g=g, m=torch.zeros(n).to(E4), v=torch.zeros(n).to(E5), m_scale=torch.zeros(n // 256, dtype=torch.uint8),
               v_scale=torch.zeros(n // 256, dtype=torch.uint8))
    row = {k: x.cuda() for k, x in row.items()}
    tsr.tsr_adamw_batched([row], 1, 1e-3)
    torch.cuda.synchronize()
    p = f64(row["p"])
    big = np.abs(f64(row["g"])) > 1e-6
    assert np.all(np.abs(p[big] + 1e-3 * np.sign(g.numpy()[big])) < 2e-5) and p[4] == 0      # the first step is lr times the sign (eps beside |g|)
    v = f64(row["v"])
    assert np.all(v[np.arange(n) != 4] > 0) and v[4] == 0 and f64(row["m"])[4] == 0
    row["g"].zero_()                                                          # a moment without its gradient: bounded by m / sqrt(v)
    tsr.tsr_adamw_batched([row], 2, 1e-3)
    torch.cuda.synchronize()
    assert np.all(np.abs(f64(row["p"]) - p) < 2e-3)


def test_8_bit_states_keep_their_mean(tsr):
    """With beta2 = 0.999 and no gradient v loses a thousandth a step, far less than half a step of its type (an eighth).
    The mean of a million values after ten steps has to be 0.999^10 of the first; the variance of one rounding is at most
    p (1 - p) (1/4)^2 with p = 0.004, so ten steps of n values leave a standard deviation of 0.05 / sqrt(n) = 5e-5."""
    n = 1 << 20
    row = dict(p=torch.zeros(n), g=torch.zeros(n), m=torch.full((n,), 256.0).to(E4), v=torch.full((n,), 32768.0).to(E5),
               m_scale=torch.full((n // 256,), 127, dtype=torch.uint8), v_scale=torch.full((n // 256,), 127, dtype=torch.uint8))
    row = {k: x.cuda() for k, x in row.items()}
    for t in range(1, 11):
        tsr.tsr_adamw_batched([row], t, 0.0, seed=7)
    torch.cuda.synchronize()
    assert abs(value_of(row, "v", n).mean() / 32768.0 - f32(0.999) ** 10) < 5e-4
    assert abs(value_of(row, "m", n).mean() / 256.0 - f32(0.9) ** 10) < 5e-4


@pytest.mark.parametrize("eps", [1e-8, 0.0])
def test_8_bit_states_of_tiny_and_of_no_gradients(tsr, eps):
    """Gradients whose squares are subnormal or vanish in fp32: the step is finite and lr times |m| / sqrt(v) at most where v is held
    in fp32; with neither gradient nor state it is nothing, or not a number where eps is 0, as the formula says."""
    n = 512
    g = torch.full((n,), 1e-21)                                               # 0.001 g^2 = 1e-45: the least subnormal number
    g[256:] = 0
    row = dict(p=torch.ones(n), g=g, m=torch.zeros(n).to(E4), v=torch.zeros(n).to(E5), m_scale=torch.zeros(2, dtype=torch.uint8), v_scale=torch.zeros(2, dtype=torch.uint8))
    row = {k: x.cuda() for k, x in row.items()}
    tsr.tsr_adamw_batched([row], 1, 1e-3, eps=eps)
    torch.cuda.synchronize()
    p = f64(row["p"])
    assert np.all(np.abs(p[:256] - 1) <= 1e-3 * 1.001)
    assert np.all(p[256:] == 1) if eps else np.all(np.isnan(p[256:]))


def test_the_same_call_gives_the_same_bits_and_another_seed_others(tsr):
    rows = [eight(70001, 40, torch.bfloat16, torch.bfloat16) for _ in range(3)]
    for r, seed in zip(rows, (5, 5, 6)):
        tsr.tsr_adamw_batched([r], 3, 1e-2, seed=seed)
    torch.cuda.synchronize()
    for k in ("p", "m", "v"):
        a, b, c = (r[k].view(torch.uint8) for r in rows)
        assert torch.equal(a, b) and not torch.equal(a, c)


def test_recorded_into_a_graph_and_on_another_stream(tsr):
    side = torch.cuda.Stream()
    rows = [[eight(9000, 50), dict(p=draw(700, 51).cuda(), g=draw(700, 52).cuda(), m=torch.zeros(700, device="cuda"), v=torch.zeros(700, device="cuda"))] for _ in range(2)]
    norm, coef = torch.zeros(2, 1, device="cuda"), torch.zeros(2, 1, device="cuda")
    sets = [tsr.TensorSet(r) for r in rows]
    ws = [tsr.workspace(tsr.tsr_grad_norm_workspace_bytes(s)) for s in sets]
    torch.cuda.synchronize()
    def step(i, stream=None):
        tsr.tsr_grad_norm_batched(sets[i], 0.5, norm[i], coef[i], ws=ws[i], stream=stream)
        tsr.tsr_adamw_batched(sets[i], 6, 1e-2, wd=0.1, g_scale=coef[i], seed=3, stream=stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        step(1, side)
        side.synchronize()
        assert torch.equal(norm[0], norm[1]) and torch.equal(coef[0], coef[1]) and coef[0].item() < 1
        for a, b in zip(rows[0], rows[1]):
            assert all(torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)) for k in ("p", "m", "v"))


# ------------------------------------------------------------------ norm
@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,shift", [([1], 0), ([0], 0), ([5, 0, 3], 1), ([512] * 17, 0), ([513] * 130, 0), ([40000, 1, 9000], 3), ([3_000_001, 7], 0)])
def test_norm(tsr, gt, sizes, shift):
    gs = [offset(draw(n, 60, j, std=1e-2).to(gt), shift)[0] for j, n in enumerate(sizes)]
    want = np.sqrt(sum(np.sum(f64(g) ** 2) for g in gs))
    norm, coef = torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")
    for top in (1e-3, 1e3):
        tsr.tsr_grad_norm_batched([dict(g=g) for g in gs], top, norm, coef)
        torch.cuda.synchronize()
        assert abs(norm.item() - want) <= 2 * U * want
        expect = 1.0 if want <= f32(top) else f32(top) / want
        assert abs(coef.item() - expect) <= 2 * U * expect
    tsr.tsr_grad_norm_batched([dict(g=g) for g in gs], 1.0, norm)
    torch.cuda.synchronize()
    assert abs(norm.item() - want) <= 2 * U * want


def test_norm_of_large_small_and_unfit_values(tsr):
    norm, coef = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    for n in (100, 100_000):
        for value, top in ((1e30, 1.0), (1e-30, 1.0)):                        # squares beyond fp32
            g = torch.full((n,), value, device="cuda")
            tsr.tsr_grad_norm_batched([dict(g=g)], top, norm, coef)
            torch.cuda.synchronize()
            want = f32(value) * np.sqrt(n)
            assert abs(norm.item() / want - 1) < 1e-6 and abs(coef.item() / min(1.0, top / want) - 1) < 1e-6
        for value in (float("nan"), float("inf")):
            g[n // 2] = value
            tsr.tsr_grad_norm_batched([dict(g=g)], float("inf"), norm, coef)
            torch.cuda.synchronize()
            assert not np.isfinite(norm.item()) and np.isnan(coef.item())
        g.fill_(2.0)
        tsr.tsr_grad_norm_batched([dict(g=g)], float("inf"), norm, coef)
        torch.cuda.synchronize()
        assert coef.item() == 1.0


def test_a_gradient_of_two_tensors(tsr):
    """Tied gradients: read twice, each tensor steps as it does alone."""
    g = si.normal((700,), si.stream_key(97, 1)).cuda()
    p = [si.normal((700,), si.stream_key(97, 2 + i)).cuda() for i in range(2)]
    alone = [x.clone() for x in p]
    state = lambda: dict(m=torch.zeros(700, device="cuda"), v=torch.zeros(700, device="cuda"))      # noqa: E731
    tsr.tsr_adamw_batched([dict(p=x, g=g, **state()) for x in p], 1, 1e-3)
    for x in alone:
        tsr.tsr_adamw_batched([dict(p=x, g=g, **state())], 1, 1e-3)
    torch.cuda.synchronize()
    assert torch.equal(p[0], alone[0]) and torch.equal(p[1], alone[1])


@pytest.mark.parametrize("t", [1, 100000])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-20, 1e-8])
def test_8_bit_states_whose_root_is_of_a_subnormal_number(tsr, t, eps):
    """Second moments around and below the least normal fp32 number, where the unit's root takes no more values.  p is 0, so
    that the step is what is seen.  Moments are computed as the kernel does, each product and sum rounded to fp32; from there on
    root and reciprocal are off by a whole step of fp32 (2 half steps each), sum, product, and the product with lr by half a one:
    7, and 1 for what is of second order and the rounding of lr."""
    n = 2048
    g = (10.0 ** (-23.0 + 6.0 * np.arange(n) / n)).astype(np.float32) * np.where(np.arange(n) % 3, 1, -1).astype(np.float32)
    row = dict(p=torch.zeros(n), g=torch.from_numpy(g), m=torch.zeros(n).to(E4), v=torch.zeros(n).to(E5), m_scale=torch.zeros(n // 256, dtype=torch.uint8),
               v_scale=torch.zeros(n // 256, dtype=torch.uint8))
    row = {k: x.cuda() for k, x in row.items()}
    tsr.tsr_adamw_batched([row], t, 1e-3, eps=eps)
    torch.cuda.synchronize()
    f = np.float32
    b1, b2 = f(0.9), f(0.999)
    m, v = g * (f(1) - b1), (g * g) * (f(1) - b2)
    c1, c2 = f(1 / (1 - float(b1) ** t)), f(1 / (1 - float(b2) ** t))
    m, v = m * c1, v * c2
    assert (v == 0).sum() > 100 and ((v > 0) & (v < 2.0 ** -126)).sum() > 500 and (v >= 2.0 ** -126).sum() > 100
    with np.errstate(divide="ignore"):
        want = -f(1e-3).astype(np.float64) * (m.astype(np.float64) / (np.sqrt(v.astype(np.float64)) + float(f(eps))))
    got = f64(row["p"])
    big = np.isinf(want) | (np.abs(want) > 3.4e38)
    assert np.array_equal(np.isinf(got), big) and np.array_equal(np.sign(got), np.sign(want))
    assert np.all(np.abs(got[~big] - want[~big]) <= 8 * U * np.abs(want[~big]))


@pytest.mark.parametrize("gt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,shift", [([32768], 0), ([32767], 1), ([1, 1023, 1024, 1025, 20000, 3], 1), ([0, 2049, 0, 5], 0), ([273] * 120, 3), ([300] * 119 + [0], 0), ([32769], 0)])
def test_norm_of_a_few_tensors_of_any_sizes(tsr, gt, sizes, shift):
    """Every element counts once: squares are whole numbers, so their sum is exact, and half a step of fp32 is left for the root
    and for the factor each (fp64 roots and quotients are off by far less)."""
    gs, total = [], 0
    for j, n in enumerate(sizes):
        x = (torch.arange(n) * 7 + j) % 13 - 6
        total += int(x.square().sum())
        gs.append(offset(x.to(gt), shift)[0])
    norm, coef = torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")
    tsr.tsr_grad_norm_batched([dict(g=g) for g in gs], 1.0, norm, coef)
    torch.cuda.synchronize()
    want = np.sqrt(float(total))
    assert abs(norm.item() - want) <= U * want * 1.0001 and abs(coef.item() - 1 / want) <= U / want * 1.0001


def test_a_run_with_8_bit_states_beside_one_with_32(tsr):
    """400 steps on the same gradients, g = size (1 + noise) of an element.  Rounding keeps the mean but for what 16 random bits
    cannot tell: each step up to 2^-16 of a step of the type is lost, a quarter of v at most, in 400 steps 400 2^-18 = 0.15 %.
    Scatter of v: a step moves a value that lies on the grid by 0.001 |g^2 - v|, so it is rounded away from it with the
    probability of that over the grid's step, at most v / 4: the variance of one rounding is at most 0.001 (g^2 + v) v / 4, of
    all that are remembered 0.0005 v^2 / (1 - 0.999^2) = v^2 / 4, the standard deviation of the mean of 2^16 ratios 0.5 / 256.
    Scatter of m: each rounding (m / 8)^2 / 4 at most, those remembered 1 / (1 - 0.9^2) of it, a standard deviation of 0.15.
    p moves along m / sqrt(v): a scatter of v with variance w <= 1/4 lengthens that by 3/8 w and terms of higher order on
    average, 0 to 20 %."""
    n, steps = 1 << 16, 400
    gen = torch.Generator(device="cuda")
    gen.manual_seed(41)
    size = torch.exp2(torch.rand(n, generator=gen, device="cuda") * 2 - 1) * 1e-3
    g = torch.zeros(n, device="cuda")
    full = dict(p=torch.zeros(n, device="cuda"), g=g, m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"))
    held = dict(p=torch.zeros(n, device="cuda"), g=g, m=torch.zeros(n).to(E4).cuda(), v=torch.zeros(n).to(E5).cuda(),
                m_scale=torch.zeros(n // 256, dtype=torch.uint8, device="cuda"), v_scale=torch.zeros(n // 256, dtype=torch.uint8, device="cuda"))
    sets = [tsr.TensorSet([full]), tsr.TensorSet([held])]
    for t in range(1, steps + 1):
        g.copy_(size * (1 + torch.randn(n, generator=gen, device="cuda")))
        for s in sets:
            tsr.tsr_adamw_batched(s, t, 1e-3, seed=17)
    torch.cuda.synchronize()
    m = (value_of(held, "m", n) - f64(full["m"])) / f64(size)
    v = value_of(held, "v", n) / f64(full["v"])
    assert abs(v.mean() - 1) <= 5 * 0.5 / 256 + 400 * 2.0 ** -18 and v.std() <= 0.5
    assert abs(m.mean()) <= 5 * 0.3 / 256                                     # |m| is twice the size at most, nearly always
    moved = f64(held["p"]).sum() / f64(full["p"]).sum()
    assert 0.98 <= moved <= 1.2, moved
