"""What the entry points on drafted tokens and on a paged cache's sequences refuse, and the sizes of their workspaces: host code, no
GPU needed.  Nothing is enqueued where an error is returned."""
import ctypes as C
import os

import pytest

from paper_2604_18002_amd import _build

A = 0x10000          # a made-up, 16-byte aligned device address: the host side never reads it
DENSE = dict(k=A, v=A, len=A, pos=None, L=2, B=3, Hkv=2, Hq=12, D=128, cap=4096)
PAGED = dict(k_pool=A, v_pool=A, pos_pool=None, table=A, len=A, free_stack=A, free_count=A, L=2, B=3, Hkv=2, Hq=12, D=128,
             page_rows=32, max_pages=64, num_pages=1000)


@pytest.fixture(scope="module")
def ngc():
    if not os.path.exists(_build.LIB_PATH):
        _build.build()
    from paper_2604_18002_amd import binding
    binding.load_library()
    return binding


def _cache(ngc, paged, **kw):
    cls, f = (ngc.ngc_paged_cache, dict(PAGED)) if paged else (ngc.ngc_cache, dict(DENSE))
    f.update(kw)
    return cls(*[f[k] for k, _ in cls._fields_])


def _attn(ngc, paged, cache=None, **kw):
    lib = ngc.load_library()
    a = dict(layer=-1, k=A, v=A, parent=A, n=None, W=8, q=A, scale=0.1, hint=0, out=A, lse=None, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    fn = lib.ngc_paged_tree_attn if paged else lib.ngc_tree_attn
    c = cache if cache is not None else _cache(ngc, paged)
    return fn(C.byref(c), a["layer"], a["k"], a["v"], a["parent"], a["n"], a["W"], a["q"], a["scale"], a["hint"], a["out"], a["lse"],
              a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("paged", [False, True])
def test_tree_attention(ngc, paged):
    for name in ("k", "v", "parent", "q", "out", "ws"):
        assert _attn(ngc, paged, **{name: None}) == ngc.NGC_EINVAL, name
    for name in ("k", "v", "q", "out", "ws"):
        assert _attn(ngc, paged, **{name: A + 8}) == ngc.NGC_EINVAL, name
    for bad in (dict(layer=2), dict(layer=-2), dict(W=0), dict(W=-4), dict(hint=-1), dict(scale=0.0), dict(scale=-0.1),
                dict(scale=float("nan")), dict(scale=float("inf"))):
        assert _attn(ngc, paged, **bad) == ngc.NGC_EINVAL, bad
    assert _attn(ngc, paged, W=65) == ngc.NGC_EUNSUPPORTED
    assert _attn(ngc, paged, ws_bytes=64) == ngc.NGC_ENOSPC
    for bad in (dict(D=96), dict(Hq=13), dict(Hq=34), dict(B=0), dict(L=0)):
        assert _attn(ngc, paged, _cache(ngc, paged, **bad)) == ngc.NGC_EINVAL, bad
    if paged:
        for bad in (dict(page_rows=48), dict(page_rows=16), dict(table=None), dict(k_pool=A + 8), dict(max_pages=0)):
            assert _attn(ngc, paged, _cache(ngc, paged, **bad)) == ngc.NGC_EINVAL, bad
    else:
        assert _attn(ngc, paged, _cache(ngc, paged, cap=1 << 24)) == ngc.NGC_EUNSUPPORTED
        assert _attn(ngc, paged, _cache(ngc, paged, k=A + 2)) == ngc.NGC_EINVAL
        assert ngc.load_library().ngc_tree_attn(None, 0, A, A, A, None, 8, A, 0.1, 0, A, None, A, 1 << 40, None) == ngc.NGC_EINVAL


def test_verification(ngc):
    lib = ngc.load_library()
    order = ("target", "draft", "stride", "token", "parent", "n", "B", "W", "V", "u", "us", "path", "n_path", "next", "ws", "ws_bytes")

    def call(**kw):
        a = dict(target=A, draft=None, stride=100, token=A, parent=A, n=None, B=3, W=8, V=100, u=A, us=A, path=A, n_path=A, next=A, ws=A,
                 ws_bytes=1 << 30)
        a.update(kw)
        return lib.ngc_tree_verify(*[a[k] for k in order], None)
    for name in ("target", "token", "parent", "u", "us", "path", "n_path", "next", "ws"):
        assert call(**{name: None}) == ngc.NGC_EINVAL, name
    for bad in (dict(B=0), dict(W=0), dict(V=0), dict(V=-1), dict(stride=99), dict(ws=A + 4), dict(target=A + 2), dict(draft=A + 1)):
        assert call(**bad) == ngc.NGC_EINVAL, bad
    assert call(W=65) == ngc.NGC_EUNSUPPORTED
    assert call(V=0x7FFFFFFF, stride=1 << 40) == ngc.NGC_EUNSUPPORTED
    assert call(ws_bytes=ngc.ngc_verify_workspace_bytes(3, 100) - 1) == ngc.NGC_ENOSPC
    assert ngc.ngc_verify_workspace_bytes(0, 5) == 0 == ngc.ngc_verify_workspace_bytes(5, 0)


@pytest.mark.parametrize("paged", [False, True])
def test_commits(ngc, paged):
    lib = ngc.load_library()

    def call(cache=None, **kw):
        a = dict(layer=-1, k=A, v=A, pos=None, path=A, n=A, W=8, ws=A, ws_bytes=1 << 30)
        a.update(kw)
        c = cache if cache is not None else _cache(ngc, paged)
        fn = lib.ngc_paged_tree_commit if paged else lib.ngc_tree_commit
        return fn(C.byref(c), a["layer"], a["k"], a["v"], a["pos"], a["path"], a["n"], a["W"], a["ws"], a["ws_bytes"], None)
    for name in ("k", "v", "path", "n", "ws"):
        assert call(**{name: None}) == ngc.NGC_EINVAL, name
    for bad in (dict(layer=2), dict(layer=-2), dict(W=0), dict(k=A + 8), dict(v=A + 4), dict(ws=A + 8)):
        assert call(**bad) == ngc.NGC_EINVAL, bad
    assert call(W=65) == ngc.NGC_EUNSUPPORTED
    assert call(ws_bytes=64) == ngc.NGC_ENOSPC
    assert call(_cache(ngc, paged, D=80)) == ngc.NGC_EINVAL
    if paged:
        assert call(ws_bytes=4 * 64 + 8 * 12 - 1) == ngc.NGC_ENOSPC
        assert call(_cache(ngc, paged, free_stack=None)) == ngc.NGC_EINVAL


def test_sequences_of_a_paged_cache(ngc):
    lib = ngc.load_library()
    need = lib.ngc_paged_pool_workspace_bytes(C.byref(_cache(ngc, True)))
    assert need >= lib.ngc_paged_workspace_bytes(C.byref(_cache(ngc, True)))
    for fn in (lib.ngc_paged_fork, lib.ngc_paged_free):
        def call(cache=None, layer=-1, mark=A, ws=A, ws_bytes=need):
            c = cache if cache is not None else _cache(ngc, True)
            return fn(C.byref(c), layer, mark, ws, ws_bytes, None)
        assert call(mark=None) == ngc.NGC_EINVAL and call(ws=None) == ngc.NGC_EINVAL and call(ws=A + 8) == ngc.NGC_EINVAL
        assert call(layer=2) == ngc.NGC_EINVAL and call(layer=-2) == ngc.NGC_EINVAL
        assert call(ws_bytes=64) == ngc.NGC_ENOSPC
        assert call(_cache(ngc, True, page_rows=33)) == ngc.NGC_EINVAL
        assert call(_cache(ngc, True, B=60000, L=60, max_pages=16384)) in (ngc.NGC_EUNSUPPORTED, ngc.NGC_ENOSPC)
        assert call(_cache(ngc, True, B=60000, L=60, max_pages=16384), ws_bytes=1 << 40) == ngc.NGC_EUNSUPPORTED
    many = _cache(ngc, True, B=8193)
    assert lib.ngc_paged_fork(C.byref(many), -1, A, A, 1 << 40, None) == ngc.NGC_EUNSUPPORTED
    compact = lambda c, ws=A, n=need: lib.ngc_paged_compact(C.byref(c), ws, n, None)     # noqa: E731
    assert compact(_cache(ngc, True), None) == ngc.NGC_EINVAL and compact(_cache(ngc, True), A + 8) == ngc.NGC_EINVAL
    assert compact(_cache(ngc, True), n=need // 100) == ngc.NGC_ENOSPC
    assert compact(_cache(ngc, True, table=None)) == ngc.NGC_EINVAL
    assert compact(_cache(ngc, True, B=60000, L=60, max_pages=16384), n=1 << 40) == ngc.NGC_EUNSUPPORTED


def test_workspaces_serve_the_cache_s_own_calls_too(ngc):
    lib = ngc.load_library()
    for B, Hkv, Hq, L, cap in ((1, 2, 8, 1, 512), (64, 2, 12, 28, 4096), (256, 4, 64, 1, 16384), (1, 1, 16, 4, 100000)):
        c = _cache(ngc, False, B=B, Hkv=Hkv, Hq=Hq, L=L, cap=cap)
        sizes = [lib.ngc_tree_workspace_bytes(C.byref(c), W) for W in (1, 8, 64)]
        assert min(sizes) >= lib.ngc_workspace_bytes(C.byref(c), 100) and max(sizes) < 1 << 30
    c = _cache(ngc, False)
    assert lib.ngc_tree_workspace_bytes(C.byref(c), 0) == 0 == lib.ngc_tree_workspace_bytes(C.byref(c), 65)
    assert lib.ngc_tree_workspace_bytes(None, 4) == 0 == lib.ngc_paged_pool_workspace_bytes(None)
    assert lib.ngc_paged_tree_workspace_bytes(C.byref(_cache(ngc, True, page_rows=40)), 4) == 0


def test_the_front_wants_tensors(ngc):
    with pytest.raises((AttributeError, TypeError)):
        ngc.ngc_tree_verify("x", None, 1, None, None, None, 1, 1, 1, None, None, None, None, None, None, stream=0)
    with pytest.raises((AttributeError, TypeError)):
        ngc.ngc_paged_compact(object(), None, stream=0)
