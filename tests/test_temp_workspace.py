"""The workspace of a call that brings none: it comes from the pool of the stream that the call's kernels run on, so the
allocator hands the block on in that stream's order, from what used it before and to what uses it next."""
import contextlib

import pytest
import torch


@pytest.fixture(scope="module")
def binding():
    from paper_2602_08007_amd import binding as b
    return b


def test_the_block_is_taken_on_the_stream_that_uses_it(binding, monkeypatch):
    """Without a GPU: which stream is current while the block is allocated."""
    class Stream:
        pass
    current, side = Stream(), Stream()
    at = [current]
    @contextlib.contextmanager
    def stream(s):
        at.append(s)
        yield
        at.pop()
    taken = []
    def workspace(nbytes, device):
        taken.append((nbytes, at[-1]))
        return torch.empty(nbytes, dtype=torch.uint8)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda x, s: None)
    monkeypatch.setattr(binding, "workspace", workspace)
    for s, expect in ((None, current), (side, side), (current, current)):
        binding._temp_workspace(512, "cpu", s)
        assert taken.pop() == (512, expect)
        assert at == [current]
    with pytest.raises(ValueError):
        binding._temp_workspace(512, "cpu", 1234)


@pytest.mark.gpu
def test_a_block_that_the_current_stream_still_uses_is_not_taken_for_another(monkeypatch):
    """Work is queued on the current stream that uses a block which Python has dropped; a call on another stream gets another."""
    import paper_2602_08007_amd as tsr
    from paper_2602_08007_amd import binding
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    a, b = (torch.randn(4_000_001, generator=gen, device="cuda") for _ in range(2))
    want = [x.double().square().sum().sqrt().item() for x in (a, b)]
    sets = [tsr.TensorSet([dict(g=x)]) for x in (a, b)]
    norm, coef = torch.zeros(2, 1, device="cuda"), torch.zeros(2, 1, device="cuda")
    ops = []
    for rows in (100, 200):
        q, s = tsr.fp8_matrix(rows, 5000)
        tsr.tsr_fp8_quantize(torch.randn(rows, 5000, generator=gen, device="cuda"), q, s)
        ops += [q, s]
    C = torch.zeros(3, 100, 200, device="cuda", dtype=torch.bfloat16)
    tsr.tsr_fp8_matmul(*ops, C[2])
    torch.cuda.synchronize()
    side, places = torch.cuda.Stream(), []
    plain = binding.workspace
    def workspace(*args):
        w = plain(*args)
        places.append((w.data_ptr(), w.data_ptr() + w.numel()))
        return w
    monkeypatch.setattr(binding, "workspace", workspace)
    for _ in range(5):
        for i, stream in enumerate((None, side)):
            tsr.tsr_grad_norm_batched(sets[i], 1.0, norm[i], coef[i], stream=stream)
            tsr.tsr_fp8_matmul(*ops, C[i], stream=stream)
        (x, y, z, w) = places
        assert all(p[1] <= q[0] or q[1] <= p[0] for p in (x, y) for q in (z, w))
        places.clear()
        torch.cuda.synchronize()
        for i in range(2):
            assert abs(norm[i].item() / want[i] - 1) <= 2.0 ** -23 and abs(coef[i].item() * want[i] - 1) <= 2.0 ** -23
            assert torch.equal(C[i], C[2])
