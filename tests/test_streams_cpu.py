"""What a call makes by itself (workspaces, outputs) is made on the call's
stream, not on torch's current one (no GPU needed)."""
import ast
import contextlib
import inspect

import pytest
import torch

from paper_2607_21291_gb300 import adadsf as A

MAKERS = {"empty", "zeros", "full", "ones", "tensor", "empty_like", "zeros_like"}


def name_of(call):
    f = call.func
    return f.attr if isinstance(f, ast.Attribute) else getattr(f, "id", "")


def test_the_binding_makes_tensors_on_the_calls_stream():
    """Every function that takes a stream hands it to workspace(), and makes other tensors under _torch_on(stream)."""
    seen = 0
    for f in ast.walk(ast.parse(inspect.getsource(A))):
        if not isinstance(f, ast.FunctionDef) or "stream" not in [a.arg for a in f.args.args]:
            continue
        under = set()
        for block in ast.walk(f):
            if isinstance(block, ast.With) and any(ast.unparse(i.context_expr) == "_torch_on(stream)" for i in block.items):
                under |= set(map(id, ast.walk(block)))
        for call in ast.walk(f):
            if not isinstance(call, ast.Call):
                continue
            if name_of(call) == "workspace":
                assert "stream" in [ast.unparse(a) for a in call.args] + [ast.unparse(k.value) for k in call.keywords], f.name
                seen += 1
            elif name_of(call) in MAKERS:
                assert id(call) in under, (f.name, ast.unparse(call))
                seen += 1
    assert seen >= 20


def test_workspace_is_cleared_on_its_stream(monkeypatch):
    now, made = [None], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def zeros(*size, **kw):
        made.append(now[-1])
        return torch.empty(*size, dtype=kw["dtype"]).zero_()

    monkeypatch.setattr(A.torch.cuda, "stream", on)
    monkeypatch.setattr(A.torch, "zeros", zeros)
    assert A.workspace(1000, "cpu").numel() == 1000
    side = Stream("side", [])
    assert A.workspace(10, "cpu", side).numel() == 256
    assert made == [None, side]


def test_a_function_without_that_is_found():
    """The first test's own check: a workspace without the stream, and a tensor outside the block."""
    for body in ("ws = workspace(10, x.device)", "out = torch.empty(3)"):
        source = f"def f(x, stream=None):\n    {body}\n"
        with pytest.MonkeyPatch.context() as m:
            m.setattr(inspect, "getsource", lambda _: source)
            with pytest.raises(AssertionError):
                test_the_binding_makes_tensors_on_the_calls_stream()


class Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append((self.name, "waits for", other.name))


class Result:
    def __init__(self, log):
        self.log = log

    def record_stream(self, stream):
        self.log.append(("result read on", stream.name))


@pytest.fixture
def streams(monkeypatch):
    log = []
    now = [Stream("current", log)]

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        log.append(("on", stream.name))
        yield
        log.append(("off", stream.name))
        now.pop()

    monkeypatch.setattr(A.torch.cuda, "stream", on)
    monkeypatch.setattr(A.torch.cuda, "current_stream", lambda: now[-1])
    return log, now[0], Stream("side", log)


def test_a_step_on_another_stream_is_in_order_with_the_current_one(streams):
    log, _, side = streams
    with A.in_order(side) as read_outside:
        log.append("work")
        read_outside(Result(log))
    assert log == [("side", "waits for", "current"), ("on", "side"), "work", ("result read on", "current"), ("off", "side"),
                   ("current", "waits for", "side")]


def test_a_step_that_fails_is_waited_for_too(streams):
    log, _, side = streams
    with pytest.raises(ValueError):
        with A.in_order(side):
            raise ValueError
    assert log[-1] == ("current", "waits for", "side")


def test_a_step_on_the_current_stream_waits_for_nothing(streams):
    log, current, _ = streams
    for stream in (None, current):
        with A.in_order(stream) as read_outside:
            read_outside(Result(log))
    assert log == []


@pytest.mark.parametrize("module", ["align", "calibrate"])
def test_steps_run_in_order(module):
    """Functions of torch work between library calls: all of what takes a caller's stream is under in_order(stream)."""
    from importlib import import_module
    source = ast.parse(inspect.getsource(import_module(f"paper_2607_21291_gb300.{module}")))
    seen = 0
    for f in source.body:
        if isinstance(f, ast.FunctionDef) and "stream" in [a.arg for a in f.args.args[len(f.args.args) - len(f.args.defaults):]]:
            work = [s for s in f.body if not (isinstance(s, ast.Expr) and isinstance(s.value, ast.Constant))]
            assert isinstance(work[0], ast.With) and ast.unparse(work[0].items[0].context_expr) == "A.in_order(stream)", f.name
            assert all(isinstance(s, ast.Return) for s in work[1:]), f.name
            seen += 1
    assert seen == {"align": 3, "calibrate": 1}[module]


def test_streams_by_handle(monkeypatch):
    """An object with a handle alone, which the library's calls take: torch's own work goes to a stream of that handle."""
    class Handle:
        cuda_stream = 4711
    made = []
    monkeypatch.setattr(A.torch.cuda, "ExternalStream", lambda handle: made.append(handle) or Stream("external", []))
    side = Stream("side", [])
    assert A._torch_stream(side) is side and made == []
    assert A._torch_stream(Handle()).name == "external" and made == [4711]
