"""Which GPU the tensor layer of the paged cache runs on, and that all tensors of a call have to be there: with tensors that only say
that they are on a GPU, and a library that only notes how it was called."""
import contextlib
import threading
import time

import pytest
import torch

from paper_2312_17238_amd import paged

PAGES, PAGE, HEADS, DIM = 8, 16, 2, 64


def on(gpu, *shape, dtype=torch.float16):
    """Zeros that say they are on that GPU."""
    kind = type("On", (torch.Tensor,), {"is_cuda": property(lambda s: True), "device": property(lambda s: torch.device("cuda", gpu)),
                                        "get_device": lambda s: gpu, "__torch_function__": torch._C._disabled_torch_function_impl})
    return torch.zeros(*shape, dtype=dtype).as_subclass(kind)


class Library:
    """Notes (entry point, stream, current GPU) of every call."""

    def __init__(self, current):
        self.calls, self.current = [], current

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args[-1], self.current[-1]))
            return 0
        return call


@pytest.fixture
def machine(monkeypatch):
    """GPU 0 is current; GPU g's current stream is 1000 g."""
    current = [0]

    @contextlib.contextmanager
    def device(g):
        current.append(g)
        yield
        current.pop()
    library = Library(current)
    step = paged.Step(2, 8, 4, 4, PAGES, PAGE, 4, HEADS, DIM, device="cpu")      # sizes come from the real library
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[-1], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda g: 1000 * g, raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(paged.B, "lib", lambda: library)
    monkeypatch.setattr(torch, "empty", lambda *shape, dtype=None, device=None: on(torch.device(device).index, *(shape[0] if isinstance(shape[0], tuple) else shape), dtype=dtype))
    return step, library


def inputs(gpu):
    i = lambda *s: on(gpu, *s, dtype=torch.int32)  # noqa: E731
    cache = paged.Cache(on(gpu, PAGES, HEADS, 1, 4, 16, 16, dtype=torch.int8), on(gpu, PAGES, HEADS, 1, DIM, 16, dtype=torch.int8),
                        on(gpu, PAGES, HEADS, dtype=torch.float32), on(gpu, PAGES, HEADS, dtype=torch.float32))
    return {"cache": cache, "ctx": i(2), "new": i(2), "table": i(2, 4), "free": i(PAGES), "count": i(1), "q": on(gpu, 8, 4, DIM), "k": on(gpu, 8, HEADS, DIM),
            "v": on(gpu, 8, HEADS, DIM), "gain": on(gpu, DIM), "freq": on(gpu, DIM // 2, dtype=torch.float32), "q_out": on(gpu, 8, 4, DIM),
            "out": on(gpu, 8, 4, DIM), "slots": i(3), "requests": i(2)}


def calls(step, x):
    return {
        "plan": lambda: step.plan(x["ctx"], x["new"], x["table"], x["free"], x["count"]),
        "write": lambda: paged.write(x["cache"], step, x["q"], x["k"], x["v"], x["gain"], x["gain"], 1e-5, x["freq"], q_out=x["q_out"]),
        "attend": lambda: paged.attend(x["cache"], step, x["q"], out=x["out"]),
        "gather": lambda: paged.gather(x["cache"], x["slots"]),
        "release": lambda: paged.release(x["requests"], PAGES, PAGE, x["ctx"], x["table"], x["free"], x["count"]),
    }


@pytest.mark.parametrize("gpu", [0, 1])
def test_calls_run_on_the_gpu_of_their_tensors(machine, gpu):
    step, library = machine
    step.device = gpu
    for name, call in calls(step, inputs(gpu)).items():
        call()
        (entry, stream, current), = library.calls
        assert name in entry and stream == 1000 * gpu and current == gpu
        library.calls.clear()
    assert library.current == [0]


USED = {"plan": ["ctx", "new", "table", "free", "count"], "write": ["cache", "q", "k", "v", "gain", "freq", "q_out"], "attend": ["cache", "q", "out"],
        "gather": ["slots"], "release": ["requests", "ctx", "table", "free", "count"]}


@pytest.mark.parametrize("name,what", [(n, w) for n, v in USED.items() for w in v])
@pytest.mark.parametrize("gpu,other", [(0, 1), (1, 0)])
def test_tensors_of_two_gpus_are_refused(machine, name, what, gpu, other):
    step, library = machine
    step.device = gpu
    x = inputs(gpu)
    calls(step, x)["plan"]()
    library.calls.clear()
    x[what] = inputs(other)[what]
    with pytest.raises(ValueError):
        calls(step, x)[name]()
    assert not library.calls


def test_two_threads_may_use_one_step(machine, monkeypatch):
    """The library reads a call's pointers while the interpreter's lock is off: another thread's call must not change them meanwhile."""
    step, _ = machine
    step.device = 0
    seen = {"plan": [], "write": [], "attend": []}

    class Slow:
        @staticmethod
        def moe_kv_plan_within(s, lists, room, plan, stream):
            a = lists._obj.ctx_len
            time.sleep(0.0005)
            seen["plan"].append((a, lists._obj.free_count))
            return 0

        @staticmethod
        def moe_kv_write(c, s, plan, rows, stream):
            a = rows._obj.q
            time.sleep(0.0005)
            seen["write"].append((a, rows._obj.inv_freq))
            return 0

        @staticmethod
        def moe_kv_attend(c, s, plan, table, query, scratch, n, stream):
            a = query._obj.q
            time.sleep(0.0005)
            seen["attend"].append((a, query._obj.out))
            return 0
    monkeypatch.setattr(paged.B, "lib", lambda: Slow)
    mine = [inputs(0) for _ in range(4)]
    calls(step, mine[0])["plan"]()
    seen["plan"].clear()

    def work(x):
        for _ in range(25):
            for name in seen:
                calls(step, x)[name]()
    threads = [threading.Thread(target=work, args=(x,)) for x in mine]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for name, (a, b) in {"plan": ("ctx", "count"), "write": ("q", "freq"), "attend": ("q", "out")}.items():
        assert sorted(seen[name]) == sorted([(x[a].data_ptr(), x[b].data_ptr()) for x in mine] * 25), name
