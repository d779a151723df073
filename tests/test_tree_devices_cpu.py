"""The tree operators in a process of several devices, without any: which device is current when the library is entered, what it sets for each."""
import os
import subprocess

import pytest
import torch

from paper_2203_16487_b200 import build, tree


class OnDevice1:
    """A tensor as the wrappers look at one, on device 1."""
    is_cuda, requires_grad, device = True, False, torch.device("cpu")       # (what the wrappers allocate beside it lands on the CPU)

    def __init__(self, shape, dtype=torch.int32):
        self.shape, self.dtype = torch.Size(shape), dtype

    def get_device(self): return 1
    def is_contiguous(self): return True
    def data_ptr(self): return 4096
    def dim(self): return len(self.shape)
    def numel(self): return self.shape.numel()
    def new_empty(self, *shape, dtype=None): return OnDevice1(shape, dtype or self.dtype)

    def stride(self, i=None):
        s = [self.shape[j + 1:].numel() for j in range(len(self.shape))]
        return tuple(s) if i is None else s[i]

    @classmethod
    def __torch_function__(cls, f, types, args=(), kwargs=None):
        assert f is torch.empty_like
        return OnDevice1(args[0].shape, (kwargs or {}).get("dtype", args[0].dtype))


class Library:
    """Notes the current device at every call that takes a stream."""

    def __init__(self, state):
        self.state, self.calls = state, []

    def __getattr__(self, name):
        if name in ("specdec_cache_scratch", "specdec_tree_attention_workspace"):
            return lambda *a: 16                               # arithmetic alone

        def call(*a):
            self.calls.append((name, self.state["current"], a[-1]))
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    state = {"current": 0}

    class Device:
        def __init__(self, d): self.d = d
        def __enter__(self): self.was, state["current"] = state["current"], self.d
        def __exit__(self, *a): state["current"] = self.was

    lib = Library(state)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(tree, "lib", lambda: lib)
    monkeypatch.setattr(tree, "_raw_stream", lambda d: {0: 0, 1: 0}[d])                 # default streams: the same handle on every device
    monkeypatch.setattr(tree, "_current_device", lambda: state["current"], raising=False)
    lib.state = state
    return lib


@pytest.mark.parametrize("current", [0, 1])
def test_every_operator_runs_on_the_tensors_device(library, current):
    library.state["current"] = current
    i32, f32 = (lambda *s: OnDevice1(s)), (lambda *s: OnDevice1(s, torch.float32))
    cache = tree.PagedCache.over(f32(2, 2, 8, 16, 4, 64), i32(3, 4), i32(3), i32(3), i32(8))
    k = f32(2, 2, 5, 4, 64)
    cache.reserve(i32(2), 5)
    cache.append(i32(2), k, k)
    cache.append(i32(2), f32(2, 5, 4, 64), f32(2, 5, 4, 64), layer=1, count=i32(2))
    cache.compact(i32(2), i32(2, 5), i32(2))
    cache.release(i32(2))
    cache.fork(i32(2), i32(2))
    tree.ancestors(i32(2, 5))
    tree.accept(i32(2, 5), i32(2, 5), i32(2, 5))
    tree.attention(f32(2, 5, 8, 64), cache, 0, i32(2), i32(2, 5, 1))
    tree.sample(f32(2, 5, 100), f32(2, 5), f32(2))
    assert len(library.calls) == 10
    for name, on, stream in library.calls:
        assert on == 1 and stream == 0, name
    assert library.state["current"] == current                # and left as it was


@pytest.fixture(scope="module")
def host_side(tmp_path_factory):
    """The operators' object files, as they are in the library, on a runtime that is tests/stub_runtime.cpp."""
    build.build()
    objs = [os.path.join(build.OBJ, n + ".o") for n in ("sample", "tree_ops", "tree_attention", "tree_attention_mma", "tree_attention_tc")]
    if not all(os.path.exists(o) for o in objs):
        build.build(force=True)
    here, exe = os.path.dirname(os.path.abspath(__file__)), str(tmp_path_factory.mktemp("stub") / "host_side")
    r = subprocess.run(["g++", "-std=c++17", "-I/usr/local/cuda/include", "-o", exe, os.path.join(here, "stub_runtime.cpp")] + objs, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    return {name: int(n) for name, n in (line.split() for line in r.stdout.splitlines())}, r.stderr


def test_shared_memory_limits_are_set_on_every_device(host_side):
    """A limit belongs to a kernel and a device: set once on each, and asked for again where it was refused."""
    assert not any(host_side[0].values()), host_side
