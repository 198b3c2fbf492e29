"""What the calls on dense parameters and 8-bit matrices refuse, on the host, before anything is launched."""
import ctypes

import pytest

FAKE = 0x10000          # never dereferenced: every call below fails its checks first
OK = 0


@pytest.fixture(scope="module")
def tsr():
    import paper_2602_08007_amd as t
    return t


def tensors(tsr, number=1, **change):
    d = (tsr.tsr_tensor_desc * number)()
    for i in range(number):
        at = FAKE + i * 0x100000
        d[i].p, d[i].g, d[i].m, d[i].v = at, at + 0x10000, at + 0x20000, at + 0x30000
        d[i].count, d[i].wd_scale = 100, 1.0
    for k, v in change.items():
        setattr(d[number - 1], k, v)
    return d


def adamw(tsr, d, count=None, t=1, beta1=0.9, beta2=0.999, eps=1e-8, hyper=True, g_scale=None):
    h = tsr.tsr_hyper(1e-3, 0.1, beta1, beta2, eps, 1.0)
    return tsr.lib.tsr_adamw_batched(d, len(d) if count is None and d is not None else count or 0, t, ctypes.byref(h) if hyper else None, 0, g_scale, None)


def test_sizes_of_the_descriptions(tsr):
    assert ctypes.sizeof(tsr.tsr_tensor_desc) == 80 and ctypes.sizeof(tsr.tsr_fp8_matrix) == 40
    assert "memory" in tsr.tsr_status_string(-7)


@pytest.mark.parametrize("change,status", [
    (dict(p=None), -1), (dict(g=None), -1), (dict(m=None), -1), (dict(v=None), -1),
    (dict(p=FAKE + 2), -1), (dict(g=FAKE + 0x10002), -1), (dict(m=FAKE + 0x20001), -1), (dict(v=FAKE + 0x30002), -1),
    (dict(p_dtype=1, p=FAKE + 1), -1), (dict(g_dtype=1, g=FAKE + 0x10001), -1),
    (dict(p_dtype=2), -3), (dict(g_dtype=3), -3), (dict(p_dtype=-1), -3), (dict(state=2), -3),
    (dict(count=-1), -2), (dict(count=(1 << 35) + 1), -2),
    (dict(state=1), -1), (dict(state=1, m_scale=FAKE + 0x40000), -1),
    (dict(p16=FAKE + 0x50001), -1), (dict(p16=FAKE + 0x50000, p_dtype=1), -1),
    (dict(wd_scale=float("nan")), -1), (dict(wd_scale=float("inf")), -1),
    # ranges that are written and meet: within a tensor, by one element, with a state's scales, with the bf16 copy
    (dict(m=FAKE), -1), (dict(v=FAKE + 0x20000 + 396), -1), (dict(p16=FAKE + 398), -1),
    (dict(state=1, m_scale=FAKE + 0x40000, v_scale=FAKE + 0x40000), -1), (dict(state=1, m_scale=FAKE + 0x20000 + 99, v_scale=FAKE + 0x40000), -1)])
def test_a_tensor_that_does_not_fit(tsr, change, status):
    assert adamw(tsr, tensors(tsr, **change)) == status


def test_tensors_that_meet_each_other(tsr):
    for change in (dict(p=FAKE), dict(p=FAKE + 396), dict(m=FAKE + 0x30000), dict(p16=FAKE + 4)):
        assert adamw(tsr, tensors(tsr, 2, **change)) == -1
    many = tensors(tsr, 200, v=FAKE + 55 * 0x100000)
    assert adamw(tsr, many) == -1


def test_the_arguments_of_a_step(tsr):
    d = tensors(tsr)
    assert adamw(tsr, None, 1) == -1
    assert adamw(tsr, d, hyper=False) == -1
    assert tsr.lib.tsr_adamw_batched(d, 0, 1, ctypes.byref(tsr.tsr_hyper()), 0, None, None) == -2
    assert tsr.lib.tsr_adamw_batched(d, -3, 1, ctypes.byref(tsr.tsr_hyper()), 0, None, None) == -2
    assert adamw(tsr, d, t=0) == -1
    assert adamw(tsr, d, beta1=1.0) == -1 and adamw(tsr, d, beta2=-0.1) == -1 and adamw(tsr, d, eps=float("nan")) == -1
    assert adamw(tsr, d, g_scale=FAKE + 1) == -1


def test_a_step_of_nothing_launches_nothing(tsr):
    d = (tsr.tsr_tensor_desc * 3)()                      # counts of zero: no pointer is needed
    assert adamw(tsr, d) == OK


def test_norm(tsr):
    f, d = tsr.lib.tsr_grad_norm_batched, tensors(tsr, 3)
    nbytes = tsr.lib.tsr_grad_norm_workspace_bytes(d, 3)
    assert nbytes >= 3 * 8 and nbytes % 256 == 0
    assert f(None, 3, 1.0, FAKE, None, FAKE, nbytes, None) == -1
    assert f(d, 0, 1.0, FAKE, None, FAKE, nbytes, None) == -2
    assert f(d, 3, 0.0, FAKE, None, FAKE, nbytes, None) == -1 and f(d, 3, float("nan"), FAKE, None, FAKE, nbytes, None) == -1
    assert f(d, 3, 1.0, None, None, FAKE, nbytes, None) == -1 and f(d, 3, 1.0, FAKE + 2, None, FAKE, nbytes, None) == -1
    assert f(d, 3, 1.0, FAKE, FAKE, FAKE, nbytes, None) == -1                    # norm and coef are two places
    assert f(d, 3, 1.0, FAKE, None, None, nbytes, None) == -1 and f(d, 3, 1.0, FAKE, None, FAKE + 8, nbytes, None) == -1
    assert f(d, 3, 1.0, FAKE, None, FAKE, 16, None) == -4
    for change, status in ((dict(count=-1), -2), (dict(g=None), -1), (dict(g_dtype=2), -3), (dict(g=FAKE + 2), -1)):
        bad = tensors(tsr, 3, **change)
        assert f(bad, 3, 1.0, FAKE, None, FAKE, 1 << 20, None) == status
        assert tsr.lib.tsr_grad_norm_workspace_bytes(bad, 3) == 0
    assert tsr.lib.tsr_grad_norm_workspace_bytes(None, 3) == 0 and tsr.lib.tsr_grad_norm_workspace_bytes(d, 0) == 0
    # the number of partial sums is bounded, whatever the tensors hold
    big = tensors(tsr, 300)
    for x in big:
        x.count = 1 << 35
    assert 0 < tsr.lib.tsr_grad_norm_workspace_bytes(big, 300) <= (4096 + 300) * 8 + 256


def test_quantize(tsr):
    def call(X=FAKE, xt=0, m=10, n=200, ldx=200, rows=1, qt=2, Q=FAKE, ldq=208, S=FAKE, lds=4, T=FAKE, ldt=16, St=FAKE, ldst=4):
        return tsr.lib.tsr_fp8_quantize(X, xt, m, n, ldx, rows, qt, Q, ldq, S, lds, T, ldt, St, ldst, None)
    for change, status in (
            (dict(X=None), -1), (dict(X=FAKE + 2), -1), (dict(X=FAKE + 1, xt=1), -1), (dict(xt=2), -3), (dict(qt=0), -3), (dict(qt=4), -3),
            (dict(m=0), -2), (dict(n=-1), -2), (dict(ldx=199), -2), (dict(rows=64), -2), (dict(rows=0), -2),
            (dict(Q=None, T=None), -1), (dict(Q=FAKE + 8), -1), (dict(ldq=200), -1), (dict(ldq=192), -2), (dict(S=None), -1), (dict(S=FAKE + 2), -1),
            (dict(lds=2), -1), (dict(lds=1), -2), (dict(T=FAKE + 1), -1), (dict(ldt=10), -1), (dict(ldt=8), -2), (dict(St=None), -1), (dict(ldst=3), -1),
            (dict(ldst=0), -2)):
        assert call(**change) == status, change


def test_matmul(tsr):
    def operand(**change):
        x = tsr.tsr_fp8_matrix(FAKE, FAKE, 208, 4, 2, 1)
        for k, v in change.items():
            setattr(x, k, v)
        return x
    def call(a=None, b=None, m=10, n=20, k=200, C=FAKE, ldc=20, ws=FAKE, nbytes=1 << 40):
        a, b = operand() if a is None else a, operand() if b is None else b
        return tsr.lib.tsr_fp8_matmul(ctypes.byref(a), ctypes.byref(b), m, n, k, C, ldc, ws, nbytes, None)
    for change, status in ((dict(m=0), -2), (dict(n=0), -2), (dict(k=0), -2), (dict(k=(1 << 22) + 1), -2), (dict(ldc=19), -2), (dict(C=None), -1), (dict(C=FAKE + 1), -1)):
        assert call(**change) == status, change
    for change, status in ((dict(q=None), -1), (dict(scale=None), -1), (dict(q=FAKE + 8), -1), (dict(ld=200), -1), (dict(ld=192), -2), (dict(scale=FAKE + 1), -1),
                           (dict(ld_scale=1), -2), (dict(ld_scale=2), -1), (dict(dtype=1), -3), (dict(dtype=4), -3), (dict(block_rows=2), -2)):
        assert call(a=operand(**change)) == status, change
        assert call(b=operand(**change)) == status, change
    assert tsr.lib.tsr_fp8_matmul(None, ctypes.byref(operand()), 10, 20, 200, FAKE, 20, None, 0, None) == -1
    assert tsr.tsr_fp8_matmul_workspace_bytes(0, 1, 1) == 0


def test_other_calls_know_nothing_of_8_bit_types(tsr):
    f = tsr.lib.tsr_project_core
    assert f(ctypes.c_void_p(FAKE), 2, 8, 8, ctypes.c_longlong(8), ctypes.c_void_p(FAKE), ctypes.c_void_p(FAKE), 4, ctypes.c_float(1.0), 0, ctypes.c_void_p(FAKE), 0,
             ctypes.c_void_p(FAKE), ctypes.c_size_t(1 << 30), None) == -3


def test_tensors_on_the_cpu_are_refused(tsr):
    import torch
    x = torch.zeros(8)
    with pytest.raises(TypeError):
        tsr.TensorSet([dict(p=x, g=x, m=x, v=x)])
    with pytest.raises(TypeError):
        tsr.tsr_fp8_quantize(torch.zeros(4, 4), *tsr.fp8_matrix(4, 4, device="cpu"))


def test_what_a_step_reads_is_not_what_it_writes(tsr):
    d = tensors(tsr, 3)
    own, other = FAKE + 0x200000, FAKE
    # the gradient: its own p (in place, or by one element at either end), another tensor's states
    for g in (own, own + 396, own - 396, own + 0x20000, other + 0x30000, other + 0x20000 + 396, other - 396):
        assert adamw(tsr, tensors(tsr, 3, g=g)) == -1, hex(g)
    assert adamw(tsr, tensors(tsr, 3, g=other + 0x40000, p16=other + 0x40000 + 396)) == -1
    # the factor: within p, the last bytes of v
    for at in (own, other + 0x30000 + 396, other + 0x20000 + 200):
        assert adamw(tsr, d, g_scale=at) == -1, hex(at)


@pytest.mark.parametrize("m,n", [((1 << 30) + 1, 64), ((1 << 31) - 1, 1), (64, (1 << 31) - 1), (1 << 28, 16), (16, (1 << 28) - 15), (1 << 21, 1 << 20)])
def test_a_product_of_too_many_rows(tsr, m, n):
    x = tsr.tsr_fp8_matrix(FAKE, FAKE, 208, 4, 2, 1)
    assert tsr.lib.tsr_fp8_matmul(ctypes.byref(x), ctypes.byref(x), m, n, 200, FAKE, 1 << 31, None, 0, None) == -2


@pytest.mark.parametrize("m,n", [((1 << 30) + 1, 1), (1, (1 << 31) - 1), (1 << 26, 1 << 12)])
def test_a_quantised_matrix_of_too_many_rows(tsr, m, n):
    assert tsr.lib.tsr_fp8_quantize(FAKE, 0, m, n, 1 << 31, 1, 2, FAKE, 1 << 31, FAKE, 1 << 24, None, 0, None, 0, None) == -2


def test_no_tensors(tsr):
    with pytest.raises(ValueError):
        tsr.TensorSet([])
    with pytest.raises(ValueError):
        tsr.tsr_adamw_batched([], 1, 1e-3)


@pytest.mark.parametrize("eps", [1e-45, 1e-39, 1.3e30, float("inf")])
def test_an_eps_that_the_step_beside_8_bit_states_cannot_take(tsr, eps):
    assert adamw(tsr, tensors(tsr, 2, state=1, m_scale=FAKE + 0x140000, v_scale=FAKE + 0x150000), eps=eps) == -1


@pytest.mark.parametrize("m,n,k", [(100, 200, 5000), (128, 128, 4100), (64, 64, 8193), (512, 512, 8192), (768, 768, 16384), (2736, 1024, 12345), (40, 4000, 1 << 20)])
def test_the_workspace_of_a_product_is_that_of_the_pieces_that_run(tsr, m, n, k):
    """Pieces begin at multiples of 512 along k, so not every number of them exists: one that does gives itself back."""
    nbytes, piece = tsr.tsr_fp8_matmul_workspace_bytes(m, n, k), m * -(-n // 4) * 16
    pieces = nbytes // piece
    assert pieces > 1 and nbytes == -(-pieces * piece // 256) * 256
    chunk = -(-(-(-k // pieces)) // 512) * 512
    assert -(-k // chunk) == pieces


@pytest.mark.parametrize("m,n,k,cut", [(16, 16, 131072, True), (300, 7, 100000, True), (32, 5461, 8192, True), (1, 5461, 2048, False), (32, 5461, 2048, False), (3, 17, 129, False)])
def test_a_long_contraction_of_few_rows_is_cut_into_pieces(tsr, m, n, k, cut):
    assert (tsr.tsr_fp8_matmul_workspace_bytes(m, n, k) > 0) == cut


def test_the_pitch_of_one_row_and_the_column_stride_of_one_column_do_not_matter(tsr):
    """Whatever torch says of them: a single row is taken with a pitch that holds it, a single column with its own."""
    import torch
    from paper_2602_08007_amd import binding
    row = torch.empty(3, 1000)[1:2, :200]
    for x, ld in ((row, 208), (torch.empty(200, 1).t(), 208), (torch.empty(200).as_strided((1, 200), (0, 1)), 208), (torch.empty(1, 7).t(), 1), (torch.empty(5, 6)[:, 2:3], 6),
                  (torch.empty(5, 6)[:, :4], 6)):
        assert binding._rows_ld(x) == ld, (x.shape, x.stride())
    for x in (torch.empty(6, 5).t(), torch.empty(6, 10)[:, ::2], torch.empty(1, 10)[:, ::2]):
        with pytest.raises(TypeError):
            binding._rows_ld(x)


def test_numbers_that_do_not_fit_an_int_are_not_cut_to_its_low_bits(tsr, monkeypatch):
    """ctypes takes the low 32 bits of a larger number: 2^32 + 4 rows would be taken as 4.  Without a GPU: tensors without storage,
    and a stand-in for the launch."""
    import torch
    from paper_2602_08007_amd import binding
    device, calls = torch.device("cuda", 0), []
    monkeypatch.setattr(binding, "_device_of", lambda *t: device)
    monkeypatch.setattr(binding, "_launch", lambda dev, stream, fn, *args: calls.append(args))
    monkeypatch.setattr(binding, "_ptr", lambda t: None if t is None else FAKE)
    monkeypatch.setattr(binding, "_temp_workspace", lambda *a: torch.empty(0))
    E4, big = torch.float8_e4m3fn, (1 << 32) + 4
    def pair(rows, cols):
        return tsr.fp8_matrix(rows, cols, E4, device="meta")
    x = torch.empty(4, 4, device="meta")
    tsr.tsr_fp8_quantize(x, *pair(4, 4))
    tsr.tsr_fp8_matmul(*pair(4, 4), *pair(4, 4), torch.empty(4, 4, dtype=torch.bfloat16, device="meta"))
    assert len(calls) == 2
    with pytest.raises(OverflowError):
        tsr.tsr_fp8_quantize(torch.empty(big, 4, device="meta"), *pair(big, 4))
    with pytest.raises(OverflowError):
        tsr.tsr_fp8_quantize(torch.empty(4, big, device="meta"), *pair(4, big))
    for m, n, k in ((big, 4, 4), (4, big, 4), (4, 4, big)):
        with pytest.raises(OverflowError):
            tsr.tsr_fp8_matmul(*pair(m, k), *pair(n, k), torch.empty(m, n, dtype=torch.bfloat16, device="meta"))
        with pytest.raises(OverflowError):
            tsr.tsr_fp8_matmul_workspace_bytes(m, n, k)
    p = torch.empty(8, device="meta")
    tsr.tsr_adamw_batched([dict(p=p, g=p, m=p, v=p)], 1, 1e-3)
    with pytest.raises(OverflowError):
        tsr.tsr_adamw_batched([dict(p=p, g=p, m=p, v=p)], (1 << 32) + 1, 1e-3)
    assert len(calls) == 3


@pytest.mark.parametrize("change", [dict(lr=float("nan")), dict(lr=float("inf")), dict(wd=float("nan")), dict(wd=-float("inf")), dict(scale=float("nan")),
                                    dict(lr=1e30, scale=1e30), dict(lr=1e30, wd=1e30)])
def test_a_step_whose_factors_are_not_finite(tsr, change):
    h = dict(lr=1e-3, wd=0.1, beta1=0.9, beta2=0.999, eps=1e-8, scale=1.0) | change
    d = tensors(tsr)
    assert tsr.lib.tsr_adamw_batched(d, 1, 1, ctypes.byref(tsr.tsr_hyper(**h)), 0, None, None) == -1
