"""Whose memory a call's own tensors are: the stream's that the call runs on, not the caller's current one.

Torch hands a block back to the stream that it was allocated on as soon as its tensor is dropped.  A workspace allocated
on the current stream for kernels of another one is overwritten while they still use it."""
import ast
import contextlib
import inspect

import pytest
import torch

import paper_2302_12510_b200 as dy
from paper_2302_12510_b200 import binding

DEV = "cuda:0"


# ---------------------------------------------------------------- on the host

def test_calls_with_a_stream_allocate_through_one_helper():
    tree = ast.parse(inspect.getsource(binding))
    taking = [f for f in tree.body if isinstance(f, ast.FunctionDef) and any(a.arg == "stream" for a in f.args.args)]
    assert len(taking) > 20
    for f in taking:
        if f.name in ("_new", "_torch_stream", "_stream"):
            continue
        for call in (n for n in ast.walk(f) if isinstance(n, ast.Call) and isinstance(n.func, ast.Attribute)):
            assert call.func.attr not in ("empty", "zeros", "empty_like", "zeros_like", "new_empty", "new_zeros", "full", "ones"), (f.name, call.lineno)
        for call in (n for n in ast.walk(f) if isinstance(n, ast.Call) and isinstance(n.func, ast.Name)):
            if call.func.id == "_new":                       # like, shape, dtype, stream
                assert isinstance(call.args[3], ast.Name) and call.args[3].id == "stream", (f.name, call.lineno)
            if call.func.id == "_workspace":                 # need, ws, like, stream
                assert isinstance(call.args[3], ast.Name) and call.args[3].id == "stream", (f.name, call.lineno)


def test_the_helper_allocates_on_the_streams_side(monkeypatch):
    current = ["mine"]

    @contextlib.contextmanager
    def on(s):
        before, current[0] = current[0], s
        yield
        current[0] = before

    class Like:
        device = DEV
        made = []

        def new_empty(self, shape, dtype=None):
            t = Like()
            t.stream, t.users = current[0], []
            t.record_stream = t.users.append
            Like.made.append(t)
            return t
        new_zeros = new_empty

    monkeypatch.setattr(binding, "_torch_stream", lambda stream, device: stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[0])
    monkeypatch.setattr(torch.cuda, "stream", on)
    for zero in (False, True):
        out = binding._new(Like(), 4, torch.uint8, "theirs", zero=zero)
        assert (out.stream, out.users) == ("theirs", ["mine"])         # returned: the caller's stream may use it, too
        ws = binding._new(Like(), 4, torch.uint8, "theirs", zero=zero, returned=False)
        assert (ws.stream, ws.users) == ("theirs", [])
        for same in ("mine", None):
            out = binding._new(Like(), 4, torch.uint8, same, zero=zero)
            assert (out.stream, out.users) == ("mine", [])


# ---------------------------------------------------------------- on the device

def calls(seed):
    """(name, f(stream)) of calls that take their outputs and workspaces from the allocator."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g).to(DEV)
    T, K, N, R, n = 700, 520, 264, 16, 3
    x, dY = r(T, K), r(T, N)
    A, B = r(n, R, K).bfloat16(), r(n, R, N).bfloat16()
    ids = (torch.arange(T, dtype=torch.int32) % (n + 1) - 1).to(DEV)
    plan = dy.AdapterPlan(ids, n)
    codes, scales = dy.dybit_checkpoint_save(x, (8, 1))
    _, v = dy.dybit_adapters(x, A, B, None, plan, want_v=True)
    pa, sa = dy.dybit_quantize_pack_2d(x, (4, 1))
    pb, sb = dy.dybit_quantize_pack_2d(r(N, K), (4, 1))
    torch.cuda.synchronize()

    def with_plan(s):
        p = dy.AdapterPlan(ids, n, stream=s)
        out = dy.dybit_adapters(x, A, B, None, p, want_v=True, stream=s)
        p.buffer.record_stream(torch.cuda.current_stream() if s is None else s)
        return out

    return [("save", lambda s: dy.dybit_checkpoint_save(x, (8, 1), stream=s)),
            ("load", lambda s: [dy.dybit_checkpoint_load(codes, K, (8, 1), scales, stream=s)]),
            ("wgrad", lambda s: [dy.dybit_checkpoint_wgrad(dY, codes, K, (8, 1), scales, stream=s)]),
            ("plan and adapters", with_plan),
            ("backward", lambda s: dy.dybit_adapters_backward(dY, codes, (8, 1), scales, A, B, None, plan, v, stream=s)),
            ("quantize", lambda s: dy.dybit_quantize_pack_2d(x, (4, 1), stream=s)),
            ("gemm", lambda s: dy.dybit_gemm(T, N, K, pa, (4, 1), sa, pb, (4, 1), sb, stream=s)[:1])]


@pytest.mark.gpu
@pytest.mark.parametrize("handle", [False, True])
def test_another_streams_call_keeps_its_memory(handle):
    work = calls(5)
    want = [[t.clone() for t in f(None)] for _, f in work]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for (name, f), w in zip(work, want):
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)                     # the call waits in line while the current stream goes on
        got = f(side.cuda_stream if handle and "plan" not in name else side)
        # the current stream takes and fills whatever the allocator has: blocks of every size that a call uses
        filled = [torch.full((1 << k,), 0x5a, dtype=torch.uint8, device=DEV) for k in range(9, 25) for _ in range(3)]
        side.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(got, w):
            assert torch.equal(a, b), name
        assert all(bool((t == 0x5a).all()) for t in filled), name
        del filled


@pytest.mark.gpu
def test_outputs_may_be_dropped_while_the_current_stream_reads_them():
    (_, save), = [c for c in calls(6) if c[0] == "save"]
    codes, scales = save(None)
    torch.cuda.synchronize()
    want = codes.clone()
    side = torch.cuda.Stream()
    got, _ = save(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(20_000_000)
    copy = got.clone()                                        # queued behind the sleep
    del got
    with torch.cuda.stream(side):
        for k in range(9, 25):
            torch.full((1 << k,), 0x5a, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    assert torch.equal(copy, want)
