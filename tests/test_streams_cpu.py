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
    assert A.workspace(10, "cpu", "side").numel() == 256
    assert made == [None, "side"]


def test_a_function_without_that_is_found():
    """The first test's own check: a workspace without the stream, and a tensor outside the block."""
    for body in ("ws = workspace(10, x.device)", "out = torch.empty(3)"):
        source = f"def f(x, stream=None):\n    {body}\n"
        with pytest.MonkeyPatch.context() as m:
            m.setattr(inspect, "getsource", lambda _: source)
            with pytest.raises(AssertionError):
                test_the_binding_makes_tensors_on_the_calls_stream()
