"""Decoder steps called from a stream that is busy, with tensors and workspaces that are dropped right behind the call: the same results as
with everything waited for."""
import pytest
import torch

from paper_2312_17238_amd import decode_loop

pytestmark = pytest.mark.gpu
NEW = ([20, 1, 33], [1, 1, 1], [2, 5, 1], [1, 1, 1])


def rows(n, seed):
    return torch.randn(n, 256, generator=torch.Generator().manual_seed(seed)).half()


def decoder():
    return decode_loop.Decoder(2, 256, 512, 4, 2, 64, 3, 80, 64, page=16)


def waited_for():
    d, outs = decoder(), []
    for i, new in enumerate(NEW):
        x, s = rows(sum(new), i).to(d.device), d.bounds(sum(new), max(new))
        torch.cuda.synchronize()
        y = d.step(s, x, new)
        torch.cuda.synchronize()
        outs.append(y.cpu())
    d.finish([0, 2])
    torch.cuda.synchronize()
    lens = d.ctx_len.tolist()
    d.close()
    return outs, lens


@pytest.mark.parametrize("side", [False, True])
def test_steps_wait_for_the_caller_and_the_caller_for_them(side):
    want, lens = waited_for()
    d, outs = decoder(), []
    inputs = [rows(sum(new), i).to(d.device) for i, new in enumerate(NEW)]
    big = torch.randn(2048, 2048, device=d.device)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream() if side else torch.cuda.current_stream()):
        for x, new in zip(inputs, NEW):
            late = torch.zeros_like(x)
            for _ in range(20):
                big = big @ big * 1e-3
            late.copy_(x)
            y = d.step(d.bounds(sum(new), max(new)), late, new)
            del late
            # what the caller's stream allocates now may lie where the rows and the step's lists were
            for n in (1 << 8, 1 << 12, 1 << 16, 1 << 20):
                torch.full((n,), 0x7F, dtype=torch.uint8, device=d.device)
            outs.append(y.clone())
            del y
            for n in (1 << 12, 1 << 15):
                torch.full((n,), 0x7F, dtype=torch.uint8, device=d.device)
        d.finish([0, 2])
        got = d.ctx_len.clone()
    torch.cuda.synchronize()
    assert got.tolist() == lens
    for a, b in zip(outs, want):
        assert torch.equal(a.cpu(), b)
    d.close()
