"""The binding's compiled argument checks give the pointers, results and refusals of the
Python ones that they stand in for."""
import importlib.util
import os

import pytest
import torch

from paper_2606_00395_amd import binding as B

pytestmark = pytest.mark.skipif(
    not os.path.exists(os.path.join(B.HERE, "_args.so")), reason="_args.so not built")


@pytest.fixture(scope="module")
def plain():
    """The binding outside its package, where no compiled module is found."""
    spec = importlib.util.spec_from_file_location("plain_binding", B.__file__)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m._torch()
    B._torch()
    assert m._need.__module__ == "plain_binding"
    assert type(B._need).__name__ == "builtin_function_or_method"
    return m


def outcome(f, *args, **kw):
    try:
        return f(*args, **kw)
    except Exception as e:
        return type(e), str(e)


X = torch.arange(12.0).reshape(3, 4)
CPU, GPU = torch.device("cpu"), torch.device("cuda", 0)
NEED = [
    ((X, "x", (3, 4)), {}),
    ((X, "x", (3, 4), torch.float32, CPU), {}),
    ((X, "x", X.shape, torch.float32, CPU, True), {}),
    ((X, "x", (3, 4), torch.float32, CPU), dict(optional=True)),
    ((X, "x", (3, 4)), dict(dtype=torch.float32, device=CPU)),
    ((X[1:], "x", (2, 4), None, CPU), {}),
    ((torch.empty(0), "x", (0,), torch.float32, CPU), {}),
    ((torch.tensor(1.0), "x", ()), {}),
    ((torch.empty(4, 0, dtype=torch.int8), "x", (4, 0), torch.int8), {}),
    # refused
    ((X, "x", (4, 3)), {}),
    ((X, "x", (3, 4, 1)), {}),
    ((X, "x", (3, -1)), {}),
    ((X, "x", (3, 1 << 70)), {}),
    ((X, "x", (3, 4), torch.bfloat16), {}),
    ((X, "x", (3, 4), torch.float32, GPU), {}),
    ((X.t(), "x", (4, 3)), {}),
    ((X[:, :2], "x", (3, 2)), {}),
    ((X.numpy(), "x", (3, 4)), {}),
    (([1.0], "x", (1,)), {}),
    ((None, "x", (3, 4)), {}),
    ((None, "x", (3, 4), None, None, False), {}),
    # absent where it may be
    ((None, "x", (3, 4), torch.float32, CPU, True), {}),
    ((None, "x", (3, 4)), dict(optional=True)),
]


@pytest.mark.parametrize("args,kw", NEED)
def test_need(plain, args, kw):
    assert outcome(B._need, *args, **kw) == outcome(plain._need, *args, **kw)


def test_need_returns_the_address(plain):
    assert B._need(X[1:], "x", (2, 4), torch.float32, CPU) == X.data_ptr() + 16


@pytest.mark.parametrize("args", [(), (X,), (X, "x")])
def test_need_without_its_arguments(plain, args):
    with pytest.raises(TypeError):
        B._need(*args)
    with pytest.raises(TypeError):
        plain._need(*args)


@pytest.mark.parametrize("x", [X, X.t(), X.to(torch.float16), X[0], X.to(torch.bfloat16),
                               torch.empty(2, 3, dtype=torch.int8)])
def test_need_act_refusals(plain, x):
    kind, text = outcome(B._need_act, x, "dy")
    assert issubclass(kind, (TypeError, ValueError)) and text
    assert (kind, text) == outcome(plain._need_act, x, "dy")
    assert outcome(B._need_act, x) == outcome(plain._need_act, x)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_need_act(plain, dtype):
    x = torch.empty((3, 5), dtype=dtype, device="cuda")
    for m in (B, plain):
        assert m._need_act(x, "x") == (3, 5, dtype, x.device)
        assert m._need(x, "x", (3, 5), dtype, x.device) == x.data_ptr()
        assert outcome(m._need, x, "x", (3, 5), dtype, CPU)[0] is ValueError


def test_tensors_without_storage_or_strides(plain):
    meta = torch.empty((3, 4), device="meta")
    sparse = torch.eye(3).to_sparse()
    for t, shape in ((meta, (3, 4)), (sparse, (3, 3))):
        got, want = outcome(B._need, t, "x", shape, torch.float32, CPU), outcome(plain._need, t, "x", shape, torch.float32, CPU)
        assert got == want and issubclass(got[0], Exception)
        assert outcome(B._need_act, t, "x") == outcome(plain._need_act, t, "x")


FIRST_CALLS = """
import builtins, threading
import torch
from paper_2606_00395_amd import binding as B

both = threading.Barrier(2)
plain_import = builtins.__import__

def slow_import(name, *args, **kw):
    if name == "torch":         # both threads are inside before either goes on
        try:
            both.wait(timeout=5)
        except threading.BrokenBarrierError:
            pass
    return plain_import(name, *args, **kw)

builtins.__import__ = slow_import
threads = [threading.Thread(target=B._torch) for _ in range(2)]
for t in threads:
    t.start()
for t in threads:
    t.join()
builtins.__import__ = plain_import
for call in (lambda: B._need(torch.zeros(3), "x", (4,)), lambda: B._need_act(torch.zeros(3), "x")):
    try:
        call()
    except ValueError as e:
        print("refused:", e)
"""


def test_first_calls_from_two_threads():
    """Threads that come to the binding first at the same time; in a process of its own, since a
    check that comes back to itself ends it."""
    import subprocess
    import sys
    root = os.path.dirname(B.HERE)
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.count("refused:") == 2, (r.returncode, r.stdout[-500:])
