"""The tree-speculation entry points without a GPU: what they refuse is refused before anything is launched, and nothing to do is done."""
import ctypes as C

import pytest
import torch

from paper_2203_16487_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def cache(**kw):
    f = dict(d_kv=4096, dtype=1, n_layers=2, n_heads=4, head_dim=64, n_pages=8, page_tokens=16, n_seqs=3, max_pages=4, stride_layer=131072, stride_side=65536,
             stride_page=4096, stride_token=256, stride_head=64, d_table=64, d_length=64, d_held=64, d_refs=64, d_status=64, d_scratch=64)
    f.update(kw)
    return C.byref(binding.Cache(**f))


def attention(**kw):
    f = dict(d_q=4096, d_out=4096, q_stride_b=2048, q_stride_t=256, q_stride_h=64, out_stride_b=2048, out_stride_t=256, out_stride_h=64, B=2, T=8, n_q_heads=4, layer=0,
             d_seqs=64, d_mask=64, mask_stride_b=8, d_n_nodes=None, max_length=0, scale=0.125, d_workspace=None, workspace_bytes=0)
    f.update(kw)
    return C.byref(binding.TreeAttentionArgs(**f))


def said(lib):
    return lib.specdec_last_error(None).decode()


BAD_CACHES = [dict(d_kv=None), dict(dtype=7), dict(n_layers=0), dict(page_tokens=12), dict(page_tokens=0), dict(head_dim=12), dict(d_kv=4104), dict(stride_token=100),
              dict(stride_head=-64), dict(d_status=None), dict(d_scratch=None), dict(max_pages=1 << 30), dict(n_seqs=0)]


@pytest.mark.parametrize("kw", BAD_CACHES)
def test_every_cache_call_refuses_a_bad_cache(lib, kw):
    c = cache(**kw)
    for call in (lambda: lib.specdec_cache_reserve(c, 64, 1, 1, None), lambda: lib.specdec_cache_release(c, 64, 1, None), lambda: lib.specdec_cache_fork(c, 64, 64, 1, None),
                 lambda: lib.specdec_cache_compact(c, 64, 1, 64, 8, 64, None), lambda: lib.specdec_cache_append(c, 64, 1, 0, 1, 4096, 4096, 8, 0, 2048, 256, 64, None, None)):
        assert call() == -1 and said(lib).startswith("cache_")


def test_cache_calls_refuse_bad_arguments(lib):
    c = cache()
    bad = [lambda: lib.specdec_cache_reserve(c, None, 1, 1, None), lambda: lib.specdec_cache_reserve(c, 64, 4, 1, None), lambda: lib.specdec_cache_reserve(c, 64, 1, -1, None),
           lambda: lib.specdec_cache_release(c, 64, -1, None), lambda: lib.specdec_cache_fork(c, 64, None, 1, None), lambda: lib.specdec_cache_compact(c, 64, 1, None, 8, 64, None),
           lambda: lib.specdec_cache_compact(c, 64, 1, 64, 0, 64, None), lambda: lib.specdec_cache_append(c, 64, 1, 2, 1, 4096, 4096, 8, 0, 2048, 256, 64, None, None),
           lambda: lib.specdec_cache_append(c, 64, 1, 0, 3, 4096, 4096, 8, 0, 2048, 256, 64, None, None), lambda: lib.specdec_cache_append(c, 64, 1, 0, 1, 4100, 4096, 8, 0, 2048, 256, 64, None, None),
           lambda: lib.specdec_cache_append(c, 64, 1, 0, 1, 4096, 4096, 8, 0, 2048, 257, 64, None, None), lambda: lib.specdec_cache_scratch(0, 1, 1)]
    for call in bad:
        assert call() == -1, said(lib)
    assert lib.specdec_cache_scratch(3, 4, 8) > 3 * 4 + 8


@pytest.mark.parametrize("kw,code", [(dict(d_q=None), -1), (dict(d_mask=None), -1), (dict(T=0), -1), (dict(B=-1), -1), (dict(layer=2), -1), (dict(n_q_heads=6), -1), (dict(scale=0.0), -1),
                                     (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(d_q=4097), -1), (dict(max_length=-1), -1), (dict(T=1025), -3)])
def test_tree_attention_refuses(lib, kw, code):
    assert lib.specdec_tree_attention(cache(), attention(**kw), None) == code and said(lib).startswith("tree_attention")


def test_tree_attention_refuses_caches_and_small_workspaces(lib):
    for kw in BAD_CACHES:
        if "d_scratch" not in kw and "n_layers" not in kw:
            assert lib.specdec_tree_attention(cache(**kw), attention(), None) in (-1, -7), kw
    assert lib.specdec_tree_attention(cache(head_dim=256, stride_head=256), attention(), None) == -7
    long = dict(page_tokens=1024, max_pages=64)
    need = lib.specdec_tree_attention_workspace(2, 8, 4, 4, 64, 1, 1024, 65536)
    assert need > 0
    for n, at in ((need - 1, 4096), (need, None), (need, 4100)):
        assert lib.specdec_tree_attention(cache(**long), attention(workspace_bytes=n, d_workspace=at), None) == -3 and "workspace" in said(lib)
    assert lib.specdec_tree_attention_workspace(2, 8, 4, 3, 64, 1, 16, 100) < 0 and lib.specdec_tree_attention_workspace(2, 8, 4, 4, 12, 1, 16, 100) < 0
    assert lib.specdec_tree_attention_workspace(0, 8, 4, 4, 64, 1, 16, 100) == 0


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_the_workspace_for_unknown_lengths_is_enough_for_any(lib, dtype):
    """max_length = 0 is "unknown" to the size function as it is to the call."""
    for B in (1, 2, 3, 7, 8, 37, 74, 128, 129):
        for T in (1, 2, 3, 5, 9, 17, 64, 200, 1024):
            for hq, hkv in ((8, 8), (32, 4), (4, 4), (37, 37), (296, 296)):
                for dim, page in ((64, 16), (128, 64), (64, 4)):
                    most = lib.specdec_tree_attention_workspace(B, T, hq, hkv, dim, dtype, page, 0)
                    for n in (1, 64, 300, 1000, 3000, 10000, 100000, 2000000, 0x7fff0000 - 1):
                        assert lib.specdec_tree_attention_workspace(B, T, hq, hkv, dim, dtype, page, n) <= most, (B, T, hq, hkv, dim, page, n)


@pytest.mark.skipif(torch.cuda.is_available(), reason="with a device the addresses would be used")
def test_unknown_lengths_pass_both_halves(lib):
    """A long cache, unknown lengths: what the size function says is what the call wants (it goes on to the launch, which fails without a device)."""
    need = lib.specdec_tree_attention_workspace(2, 8, 4, 4, 64, 1, 1024, 0)
    long = cache(page_tokens=1024, max_pages=64)
    assert need > 0 and lib.specdec_tree_attention(long, attention(workspace_bytes=need, d_workspace=4096), None) == -5, said(lib)


def test_trees_and_sample_refuse(lib):
    assert lib.specdec_tree_ancestors(None, None, 1, 8, 64, 64, None) == -1 and lib.specdec_tree_ancestors(64, None, 1, 8, None, None, None) == -1
    assert lib.specdec_tree_ancestors(64, None, 1, 0, 64, 64, None) == -1 and lib.specdec_tree_ancestors(64, None, 1, 1025, 64, 64, None) == -3
    assert lib.specdec_tree_accept(64, 64, None, None, 1, 8, 64, 64, 64, None) == -1
    s = lambda **kw: lib.specdec_sample(*{**dict(l=64, dt=0, stride=100, rows=1, V=100, u=64, t=None, k=None, p=None, m=None, per=1, tok=64, lp=None, st=None), **kw}.values())  # noqa: E731
    for kw, code in ((dict(l=None), -1), (dict(u=None), -1), (dict(tok=None), -1), (dict(V=0), -1), (dict(rows=-1), -1), (dict(per=0), -1), (dict(dt=3), -1), (dict(l=66), -1), (dict(V=262145), -3)):
        assert s(**kw) == code and said(lib).startswith("sample")


def test_nothing_to_do(lib):
    c = cache()
    assert lib.specdec_cache_reserve(c, None, 0, 1, None) == 0 and lib.specdec_cache_release(c, None, 0, None) == 0 and lib.specdec_cache_fork(c, None, None, 0, None) == 0
    assert lib.specdec_cache_compact(c, None, 0, None, 8, None, None) == 0 and lib.specdec_cache_append(c, None, 0, 0, 1, None, None, 8, 0, 0, 0, 0, None, None) == 0
    assert lib.specdec_tree_ancestors(None, None, 0, 8, None, None, None) == 0 and lib.specdec_tree_accept(None, None, None, None, 0, 8, None, None, None, None) == 0
    assert lib.specdec_sample(None, 0, 100, 0, 100, None, None, None, None, None, 1, None, None, None) == 0
    assert lib.specdec_tree_attention(c, attention(B=0, d_q=None, d_out=None, d_seqs=None, d_mask=None), None) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="with a device the addresses would be used")
def test_without_a_device_every_call_fails(lib):
    c = cache()
    for rc in (lib.specdec_cache_reserve(c, 64, 1, 1, None), lib.specdec_tree_ancestors(64, None, 1, 8, 64, 64, None), lib.specdec_tree_attention(c, attention(), None),
               lib.specdec_sample(64, 0, 100, 1, 100, 64, None, None, None, None, 1, 64, None, None)):
        assert rc == -5, said(lib)
