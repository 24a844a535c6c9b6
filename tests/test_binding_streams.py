"""What a wrapper allocates belongs to the stream that its kernels go to.  torch's allocator hands a block that was freed on a stream out
again to that stream at once, since its order keeps the old and the new use apart; kernels on another stream have no such order to
what is still queued.  So a tensor for `stream` is allocated with that stream current, and marked as in use on the caller's."""
import contextlib

import pytest
import torch

from paper_2604_27089_amd import binding as sp


@pytest.fixture
def allocations(monkeypatch):
    """(stream that was current, streams that the tensor was marked for) of every torch.empty."""
    seen, current = [], ["caller's"]

    class Tensor:
        def __init__(self):
            self.marked = []
            seen.append((current[-1], self.marked))

        def record_stream(self, stream):
            self.marked.append(stream)

    @contextlib.contextmanager
    def use(stream):
        current.append(stream)
        yield
        current.pop()

    monkeypatch.setattr(torch, "empty", lambda *a, **k: Tensor())
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    return seen


def test_tensors_belong_to_the_stream_that_is_given(allocations):
    sp._new("side", (4, 4), torch.bfloat16, "cuda")
    sp._workspace(1 << 20, "cuda", "side")
    assert [where for where, _ in allocations] == ["side", "side"]
    assert all("caller's" in marked for _, marked in allocations)


def test_without_a_stream_they_belong_to_the_current_one(allocations):
    sp._new(None, (4, 4), torch.bfloat16, "cuda")
    sp._workspace(1 << 20, "cuda")
    assert allocations == [("caller's", []), ("caller's", [])]


@pytest.mark.gpu
def test_a_block_still_in_use_is_not_taken_for_another_stream(monkeypatch):
    """The caller's stream is busy and will write to a block that is already free again; calls on another stream get other memory for
    their results and for the workspace that nobody sees."""
    M, N, K = 128, 4096, 14336
    x, w = (torch.randn(r, K, device="cuda").to(torch.bfloat16) for r in (M, N))
    (a, a_scale, _, _), (b, b_scale, _, _) = sp.sp_fp8_quant(x), sp.sp_fp8_quant(w)
    need = sp.sp_fp8_matmul_workspace_bytes(M, N, K)
    assert need > 0
    want = sp.sp_fp8_matmul(a, a_scale, b, b_scale)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    workspaces, plain = [], sp._workspace
    monkeypatch.setattr(sp, "_workspace", lambda *args: workspaces.append(plain(*args)) or workspaces[-1])
    torch.cuda._sleep(200_000_000)
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (a.numel(), a_scale.numel(), M * N * 2, need)]
    taken = {t.untyped_storage().data_ptr() for t in blocks}
    for t in blocks:
        t.fill_(0xFF)
    del blocks, t
    q, q_scale, _, _ = sp.sp_fp8_quant(x, stream=side)
    out = sp.sp_fp8_matmul(q, q_scale, b, b_scale, stream=side)
    side.synchronize()
    assert not taken & {t.untyped_storage().data_ptr() for t in (q, q_scale, out, *workspaces)}
    assert len(workspaces) == 1
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert torch.equal(q.view(torch.uint8), a.view(torch.uint8)) and torch.equal(q_scale[:, :M].view(torch.uint8), a_scale[:, :M].view(torch.uint8))
