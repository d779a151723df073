"""Beam search and the cache in 4 bits without a GPU: what the entry points refuse is refused before anything is launched, nothing to do is done, and every call runs on its tensors' device."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2203_16487_b200 import beam, binding, build, fp4, tree
from tests.test_tree_cabi_cpu import cache as full_cache
from tests.test_tree_devices_cpu import OnDevice1, library  # noqa: F401


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def said(lib):
    return lib.specdec_last_error(None).decode()


def cache(**kw):
    f = dict(d_kv=4096, dtype=3, n_layers=2, n_heads=4, head_dim=64, n_pages=8, page_tokens=16, n_seqs=3, max_pages=4, stride_layer=32768, stride_side=16384, stride_page=2048, stride_token=32,
             stride_head=512, d_table=64, d_length=64, d_held=64, d_refs=64, d_status=64, d_scratch=64)
    g = dict(d_scales=4096, scale_stride_layer=4096, scale_stride_side=2048, scale_stride_page=256, scale_stride_head=64, d_unit=None)
    for k, v in kw.items():
        (f if k in f else g)[k] = v
    return C.byref(binding.Fp4Cache(binding.Cache(**f), **g))


def tokens(**kw):
    f = dict(d_seqs=64, d_k=4096, d_v=4096, d_some=None, stride_layer=0, stride_seq=2048, stride_token=256, stride_head=64, n=1, layer=0, n_layers=1, dtype=1, T=8)
    f.update(kw)
    return C.byref(binding.PackedTokens(**f))


def attention(**kw):
    f = dict(d_q=4096, d_out=4096, q_stride_b=2048, q_stride_t=256, q_stride_h=64, out_stride_b=2048, out_stride_t=256, out_stride_h=64, B=2, T=8, n_q_heads=4, layer=0,
             d_seqs=64, d_mask=64, mask_stride_b=8, d_n_nodes=None, max_length=0, scale=0.125, d_workspace=None, workspace_bytes=0)
    f.update(kw)
    return C.byref(binding.TreeAttentionArgs(**f))


BAD = [dict(d_kv=None), dict(d_scales=None), dict(dtype=1), dict(n_layers=0), dict(page_tokens=8), dict(page_tokens=24), dict(head_dim=32), dict(head_dim=96), dict(d_kv=4104), dict(d_scales=4100),
       dict(stride_page=100), dict(scale_stride_head=-64), dict(scale_stride_page=8), dict(d_unit=66), dict(max_pages=1 << 28), dict(d_status=None)]


@pytest.mark.parametrize("kw", BAD)
def test_every_call_refuses_what_is_no_cache_in_4_bits(lib, kw):
    c = cache(**kw)
    for call in (lambda: lib.specdec_packed_cache_reserve(c, 64, 1, 1, None), lambda: lib.specdec_packed_cache_release(c, 64, 1, None), lambda: lib.specdec_packed_cache_fork(c, 64, 64, 1, None),
                 lambda: lib.specdec_packed_cache_compact(c, 64, 1, 64, 8, 64, None), lambda: lib.specdec_packed_cache_reorder(c, 64, 64, 2, 2, None),
                 lambda: lib.specdec_packed_cache_append(c, tokens(), None), lambda: lib.specdec_packed_cache_read(c, tokens(), None), lambda: lib.specdec_packed_attention(c, attention(), 1, None)):
        assert call() == -1 and said(lib).startswith("packed_")


def test_bad_arguments_are_refused(lib):
    c, f = cache(), full_cache()
    for call in (lambda: lib.specdec_packed_cache_reserve(c, 64, 4, 1, None), lambda: lib.specdec_packed_cache_reorder(c, 64, 64, 3, 2, None), lambda: lib.specdec_packed_cache_reorder(c, 64, None, 2, 2, None),
                 lambda: lib.specdec_packed_cache_reorder(c, 64, 64, 2, 0, None), lambda: lib.specdec_packed_cache_reorder(c, 64, 64, 6, 2, None), lambda: lib.specdec_cache_reorder(f, 64, 64, 3, 2, None),
                 lambda: lib.specdec_cache_reorder(f, None, 64, 2, 2, None), lambda: lib.specdec_cache_reorder(f, 64, 64, -2, 2, None)):
        assert call() == -1, said(lib)
    for kw in (dict(d_k=None), dict(d_seqs=None), dict(n=4), dict(n=-1), dict(T=-1), dict(layer=2), dict(layer=-1), dict(n_layers=3), dict(n_layers=0), dict(dtype=3), dict(d_k=4100), dict(stride_token=257)):
        assert lib.specdec_packed_cache_append(c, tokens(**kw), None) == -1, kw
        if kw != dict(n=4):                                    # (reading takes a sequence more than once)
            assert lib.specdec_packed_cache_read(c, tokens(**kw), None) == -1, kw
    assert lib.specdec_packed_cache_append(c, None, None) == -1 and lib.specdec_packed_cache_read(c, None, None) == -1
    for kw, code in ((dict(d_q=None), -1), (dict(T=0), -1), (dict(layer=2), -1), (dict(n_q_heads=6), -1), (dict(scale=0.0), -1), (dict(scale=float("nan")), -1), (dict(d_q=4097), -1), (dict(T=1025), -3)):
        assert lib.specdec_packed_attention(c, attention(**kw), 1, None) == code and said(lib).startswith("packed_attention"), kw
    assert lib.specdec_packed_attention(c, attention(), 3, None) == -1


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_the_workspace_for_unknown_lengths_is_enough_for_any(lib, dtype):
    for B in (1, 2, 3, 8, 37, 128, 129):
        for T in (1, 2, 3, 5, 9, 17, 64, 200, 1024):
            for hq, hkv in ((8, 8), (32, 4), (4, 4), (296, 296)):
                for dim in (64, 128):
                    most = lib.specdec_packed_attention_workspace(B, T, hq, hkv, dim, dtype, 16, 0)
                    assert most >= 0
                    for n in (1, 64, 300, 1000, 3000, 10000, 100000, 2000000, 0x7fff0000 - 1):
                        assert lib.specdec_packed_attention_workspace(B, T, hq, hkv, dim, dtype, 16, n) <= most, (B, T, hq, hkv, dim, n)
    assert lib.specdec_packed_attention_workspace(2, 8, 4, 4, 80, dtype, 16, 100) < 0 and lib.specdec_packed_attention_workspace(2, 8, 4, 4, 64, dtype, 8, 100) < 0


def select(**kw):
    f = dict(d_logits=64, d_scores=64, d_finished=None, d_norm=None, d_out_scores=64, d_out_parent=64, d_out_token=64, d_workspace=64, workspace_bytes=1 << 40, stride=100, dtype=0, B=2, K=4, V=100, n=4,
             end_token=0)
    f.update(kw)
    return C.byref(binding.BeamSelectArgs(**f))


def test_select_refuses(lib):
    for kw, code in ((dict(d_logits=None), -1), (dict(d_scores=None), -1), (dict(d_out_token=None), -1), (dict(B=-1), -1), (dict(K=0), -1), (dict(V=0), -1), (dict(n=0), -1), (dict(dtype=3), -1),
                     (dict(d_logits=66), -1), (dict(stride=-100), -1), (dict(K=65), -3), (dict(n=65), -3), (dict(V=(1 << 20) + 1), -3), (dict(B=20000), -3), (dict(d_workspace=None), -3),
                     (dict(d_workspace=68), -3), (dict(workspace_bytes=100), -3)):
        assert lib.specdec_beam_select(select(**kw), None) == code and said(lib).startswith("beam_select"), kw
    assert lib.specdec_beam_select(None, None) == -1
    assert lib.specdec_beam_select_workspace(2, 4, 100, 4, 3) == -1 and lib.specdec_beam_select_workspace(2, 65, 100, 4, 0) == -3


def test_nothing_to_do(lib):
    c = cache()
    assert lib.specdec_packed_cache_reserve(c, None, 0, 1, None) == 0 and lib.specdec_packed_cache_reorder(c, None, None, 0, 4, None) == 0 and lib.specdec_cache_reorder(full_cache(), None, None, 0, 4, None) == 0
    for kw in (dict(n=0, d_seqs=None, d_k=None, d_v=None), dict(T=0, d_k=None, d_v=None)):
        assert lib.specdec_packed_cache_append(c, tokens(**kw), None) == 0 and lib.specdec_packed_cache_read(c, tokens(**kw), None) == 0
    assert lib.specdec_packed_attention(c, attention(B=0, d_q=None, d_out=None, d_seqs=None, d_mask=None), 1, None) == 0
    assert lib.specdec_beam_select(select(B=0, d_logits=None, d_scores=None, d_workspace=None), None) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="with a device the addresses would be used")
def test_without_a_device_every_call_fails(lib):
    c = cache()
    for rc in (lib.specdec_packed_cache_reserve(c, 64, 1, 1, None), lib.specdec_packed_cache_append(c, tokens(), None), lib.specdec_packed_cache_read(c, tokens(), None),
               lib.specdec_packed_cache_reorder(c, 64, 64, 2, 2, None), lib.specdec_cache_reorder(full_cache(), 64, 64, 2, 2, None), lib.specdec_packed_attention(c, attention(), 1, None),
               lib.specdec_beam_select(select(), None)):
        assert rc == -5, said(lib)


class Bytes1(OnDevice1):
    """... of any type and layout; what the wrappers make of it is on device 1 too."""

    def as_strided(self, shape, stride, offset=0): return Bytes1(shape, self.dtype)
    def view(self, dtype): return Bytes1(self.shape, dtype)
    def new_empty(self, *shape, dtype=None): return Bytes1(shape[0] if isinstance(shape[0], tuple) else shape, dtype or self.dtype)


@pytest.mark.parametrize("current", [0, 1])
def test_every_operator_runs_on_the_tensors_device(library, monkeypatch, current):  # noqa: F811
    monkeypatch.setattr(beam, "_workspaces", {})
    library.state["current"] = current
    i32, f32 = (lambda *s: OnDevice1(s)), (lambda *s: Bytes1(s, torch.float32))
    books = i32(3, 4), i32(3), i32(3), i32(8)
    small = fp4.Fp4Cache.over(Bytes1((2, 2, 8, 4, 16, 32), torch.uint8), Bytes1((2, 2, 8, 4, 16, 4), torch.float8_e4m3fn), *books)
    full = tree.PagedCache.over(f32(2, 2, 8, 16, 4, 64), *books)
    k = f32(2, 2, 5, 4, 64)
    small.reserve(i32(2), 5)
    small.append(i32(2), k, k)
    small.append(i32(2), f32(2, 5, 4, 64), f32(2, 5, 4, 64), layer=1, count=i32(2))
    small.read(i32(2), 5, start=i32(2))
    small.compact(i32(2), i32(2, 5), i32(2))
    small.release(i32(2))
    small.fork(i32(2), i32(2))
    small.reorder(i32(1, 2), i32(1, 2))
    full.reorder(i32(1, 2), i32(1, 2))
    tree.attention(f32(2, 5, 8, 64), small, 0, i32(2), i32(2, 5, 1))
    beam.select(f32(2, 5, 100), f32(2, 5), 4)
    calls = [c for c in library.calls if not c[0].endswith("_workspace")]                  # (arithmetic alone)
    assert len(calls) == 11 and sum(name.startswith("specdec_packed_") for name, _, _ in calls) == 9
    for name, on, stream in calls:
        assert on == 1 and stream == 0, name
    assert library.state["current"] == current                # and left as it was


def test_shared_memory_limits_are_set_on_every_device(tmp_path):
    """The object files as they are in the library, on a runtime that is tests/stub_runtime.cpp: a limit belongs to a kernel and a device."""
    build.build()
    objs = [os.path.join(build.OBJ, n + ".o") for n in ("beam", "cache_pages", "fp4_cache", "fp4_attention", "fp4_attention_tc", "tree_attention", "tree_attention_mma", "tree_attention_tc", "tree_ops", "sample")]
    if not all(os.path.exists(o) for o in objs):
        build.build(force=True)
    here, exe = os.path.dirname(os.path.abspath(__file__)), str(tmp_path / "host_side")
    r = subprocess.run(["g++", "-std=c++17", "-I/usr/local/cuda/include", "-o", exe, os.path.join(here, "stub_beam.cpp")] + objs, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    found = {name: int(n) for name, n in (line.split() for line in r.stdout.splitlines())}
    assert len(found) == 8 and not any(found.values()), (found, r.stderr)
