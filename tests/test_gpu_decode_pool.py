"""Decoder steps with rows that belong to no request, and steps that the pool cannot serve."""
import pytest
import torch

from paper_2312_17238_amd import decode_loop

pytestmark = pytest.mark.gpu


def rows(n, seed):
    return torch.randn(n, 256, generator=torch.Generator().manual_seed(seed)).half().cuda()


def decoder(cache_slots=3, **k):
    return decode_loop.Decoder(2, 256, 512, 4, 2, 64, 3, 80, 64, page=16, cache_slots=cache_slots, **k)


def dirty():
    """Memory that torch hands out next holds NaN."""
    for n in (1 << 9, 1 << 12, 1 << 15, 1 << 18):
        for _ in range(4):
            torch.full((n,), float("nan"), dtype=torch.float16, device="cuda:0")


def test_stepping_on_after_a_request_is_finished():
    """With one request at no tokens the last row is nobody's: it comes back as it is, takes no expert, and the others get what they get in
    a step without it."""
    results = []
    for tight in (False, True):
        d = decoder()
        prompt = [20, 7, 3]
        x = d.step(d.bounds(30, 20), rows(30, 1), prompt)
        d.finish([1])
        one = d.bounds(2 if tight else 3, 1)
        x = rows(3, 2)
        with torch.cuda.stream(d.stack.compute):
            dirty()
        torch.cuda.synchronize()
        for i in range(4):
            y = d.step(one, x[:2].contiguous() if tight else x, [1, 0, 1] if i == 0 else None)
            if not tight:
                assert torch.equal(y[2], x[2])
            x = y
        d.stack.synchronize()
        assert d.ctx_len.tolist() == [24, 0, 7] and d.free_count.item() == 15 - 2 - 1
        results.append((x[:2].cpu(), d.stack.stats()))
        d.close()
    assert torch.isfinite(results[0][0]).all()
    # a product of three rows may be summed in another order than one of two: a rounding of fp16 here and there, four steps long
    assert (results[0][0].float() - results[1][0].float()).abs().max() <= 2.0 ** -6
    assert [s["needed"] for s in results[0][1]] == [s["needed"] for s in results[1][1]]


def test_a_step_without_tokens_changes_nothing():
    d = decoder()
    d.step(d.bounds(30, 20), rows(30, 1), [20, 7, 3])
    d.stack.synchronize()
    before, x = d.stack.stats(), rows(3, 2)
    y = d.step(d.bounds(3, 1), x, [0, 0, 0])
    torch.cuda.synchronize()
    assert torch.equal(x, y) and d.ctx_len.tolist() == [20, 7, 3] and d.stack.stats() == before
    d.close()


@pytest.mark.parametrize("new,what", [([1, 1, 1], "free"), ([70, 1, 1], "beyond"), ([1, 1], "fit"), ([1, -1, 1], "fit"), ([81, 0, 0], "fit"),
                                      ([40, 40, 1], "fit")])
def test_a_step_that_cannot_serve_everybody_is_refused_before_it_runs(new, what):
    """A request that was turned down would go on with a hidden state that its token is not part of."""
    d = decoder(n_pages=5)
    d.step(d.bounds(49, 33), rows(49, 1), [16, 33, 0])      # three pages of 16 and one: one is left
    d.stack.synchronize()
    before = d.ctx_len.tolist(), d.free_count.item(), d.block_table.tolist(), d.stack.stats()
    s = d.bounds(80, 80)
    with pytest.raises(ValueError, match=what):
        d.step(s, rows(80, 2), new)
    torch.cuda.synchronize()
    assert (d.ctx_len.tolist(), d.free_count.item(), d.block_table.tolist(), d.stack.stats()) == before
    # what fits is served: a page for the first request, room in the second's last one
    y = d.step(d.bounds(2, 1), rows(2, 3), [1, 1, 0])
    torch.cuda.synchronize()
    assert torch.isfinite(y).all() and d.ctx_len.tolist() == [17, 34, 0] and d.free_count.item() == 0
    d.finish([1])
    d.step(d.bounds(1, 1), rows(1, 4), [0, 0, 1])
    torch.cuda.synchronize()
    assert d.ctx_len.tolist() == [17, 0, 1] and d.free_count.item() == 2
    d.close()
