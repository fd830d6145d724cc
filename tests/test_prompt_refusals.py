"""Arguments that the calls on prompts and latent caches refuse, on the host, before anything is enqueued."""
import ctypes as C
import os

import pytest

from paper_2604_18002_amd import _build

A = 0x10000                      # a made-up, 16-byte aligned device address: the host side never reads it


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_build.LIB_PATH):
        _build.build()
    from paper_2604_18002_amd import binding
    return binding.load_library()


def cache(**kw):
    from paper_2604_18002_amd import binding
    f = dict(k_pool=A, v_pool=A, pos_pool=None, table=A, len=A, free_stack=A, free_count=A,
             L=2, B=3, Hkv=2, Hq=12, D=128, page_rows=32, max_pages=64, num_pages=1000)
    f.update(kw)
    return binding.ngc_paged_cache(*[f[k] for k, _ in binding.ngc_paged_cache._fields_])


def latent(**kw):
    return cache(**{**dict(v_pool=None, Hkv=1, Hq=16, D=576), **kw})


EINVAL, ENOSPC, EUNSUPPORTED = -1, -2, -4
WS = 1 << 40


def test_latent_caches_that_are_none(lib):
    def attn(pc):
        return lib.ngc_latent_attn(C.byref(pc), 0, None, 1, A, 0.1, 0, A, None, A, 16, None)
    assert attn(latent()) == ENOSPC                     # all that is wrong with this one is the workspace
    assert attn(latent(D=288)) == ENOSPC
    for bad in (dict(D=128), dict(D=512), dict(v_pool=A), dict(Hkv=2), dict(k_pool=None), dict(k_pool=A + 8), dict(page_rows=16),
                dict(page_rows=48), dict(len=None), dict(table=None), dict(free_stack=None), dict(Hq=0), dict(B=0), dict(num_pages=0)):
        assert attn(latent(**bad)) == EINVAL, bad
        assert lib.ngc_latent_workspace_bytes(C.byref(latent(**bad)), 1) == 0
    assert attn(latent(Hq=129)) == EUNSUPPORTED
    assert attn(latent(max_pages=16385)) == EUNSUPPORTED
    assert attn(cache()) == EINVAL


def test_attention_arguments(lib):
    pc = latent()
    def attn(layer=0, W=1, q=A, scale=0.1, hint=0, out=A, ws=A, ws_bytes=16):
        return lib.ngc_latent_attn(C.byref(pc), layer, None, W, q, scale, hint, out, None, ws, ws_bytes, None)
    assert attn() == ENOSPC
    for bad in (dict(layer=2), dict(layer=-2), dict(W=0), dict(q=None), dict(q=A + 8), dict(out=None), dict(out=A + 2), dict(ws=None),
                dict(ws=A + 4), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=3.0e38), dict(scale=float("inf")),
                dict(hint=-1)):
        assert attn(**bad) == EINVAL, bad
    assert attn(W=1025) == EUNSUPPORTED
    assert lib.ngc_latent_workspace_bytes(C.byref(pc), 0) == 0
    assert lib.ngc_latent_workspace_bytes(C.byref(pc), 1025) == 0
    sizes = [lib.ngc_latent_workspace_bytes(C.byref(pc), W) for W in (1, 2, 8, 64, 1024)]
    assert sizes[0] > 0 and sizes == sorted(sizes)      # what serves more tokens serves fewer


def test_extend_arguments(lib):
    for pc in (cache(), latent()):
        def extend(layer=-1, T=8, slot=A, start=A, ws=A, ws_bytes=16, pc=pc):
            return lib.ngc_paged_extend(C.byref(pc), layer, None, T, slot, start, ws, ws_bytes, None)
        assert extend() == ENOSPC
        for bad in (dict(layer=2), dict(T=0), dict(slot=None), dict(start=None), dict(ws=None), dict(ws=A + 8)):
            assert extend(**bad) == EINVAL, bad
        assert extend(T=(1 << 20) + 1, ws_bytes=WS) == EUNSUPPORTED
    def pool(**kw):
        return lib.ngc_paged_extend(C.byref(cache(**kw)), -1, None, 8, A, A, A, WS, None)
    assert pool(num_pages=1 << 26) == EUNSUPPORTED      # slots of 32 bits
    assert pool(L=60000, B=4, max_pages=16384) == EUNSUPPORTED       # sums of pages of 32 bits
    assert pool(D=96) == EINVAL and pool(Hq=33) == EINVAL


def test_fill_arguments(lib):
    def fill(pc, layer=0, k=A, v=A, slot=A, T=8, ws=A, ws_bytes=16):
        return lib.ngc_paged_fill(C.byref(pc), layer, k, v, None, slot, T, ws, ws_bytes, None)
    assert fill(cache()) == ENOSPC and fill(latent(), v=None) == ENOSPC
    assert fill(cache(), v=None) == EINVAL and fill(latent(), v=A) == EINVAL     # one tensor for each pool
    for bad in (dict(layer=5), dict(k=None), dict(k=A + 4), dict(v=A + 8), dict(slot=None), dict(T=0), dict(ws=None)):
        assert fill(cache(), **bad) == EINVAL, bad
    assert fill(cache(num_pages=1 << 26), ws_bytes=WS) == EUNSUPPORTED


def test_calls_that_move_or_read_two_pools_refuse_one(lib):
    pc = latent()
    p = C.byref(pc)
    assert lib.ngc_paged_append(p, 0, A, A, None, A, WS, None) == EINVAL
    assert lib.ngc_paged_decode_attn(p, 0, A, 0.1, 0, A, None, A, WS, None) == EINVAL
    assert lib.ngc_paged_score_keys(p, 0, A, None, 1, 0.1, 0, 32, A, A, WS, None) == EINVAL
    assert lib.ngc_paged_tree_attn(p, 0, A, A, A, None, 4, A, 0.1, 0, A, None, A, WS, None) == EINVAL
    assert lib.ngc_paged_tree_commit(p, 0, A, A, None, A, A, 4, A, WS, None) == EINVAL
    assert lib.ngc_paged_fork(p, -1, A, A, WS, None) == EINVAL
    assert lib.ngc_paged_compact(p, A, WS, None) == EINVAL
    assert lib.ngc_paged_free(p, -1, A, A, 16, None) == ENOSPC       # takes either kind


def test_replay_arguments(lib):
    def forward(q=A, kv=A, rope=A, stride=64, B=2, T=100, H=4, D=128, scale=0.1, out=A):
        return lib.ngc_latent_replay_attn(q, kv, rope, stride, None, None, B, T, H, D, scale, out, None, None)

    def backward(q=A, kv=A, rope=A, stride=64, B=2, T=100, H=4, D=128, scale=0.1, out=A, lse=A, dout=A, dq=A, dkv=A, drope=A, ws=A, ws_bytes=16):
        return lib.ngc_latent_replay_attn_backward(q, kv, rope, stride, None, None, out, lse, dout, B, T, H, D, scale, dq, dkv, drope, ws,
                                                   ws_bytes, None)
    assert backward() == ENOSPC
    shared = [dict(q=None), dict(q=A + 8), dict(kv=None), dict(kv=A + 2), dict(rope=None), dict(rope=A + 8), dict(out=None), dict(out=A + 8),
              dict(stride=56), dict(stride=68), dict(stride=0), dict(B=0), dict(T=0), dict(H=0), dict(D=96), dict(D=0), dict(scale=0.0),
              dict(scale=-0.1), dict(scale=float("nan")), dict(scale=float("inf"))]
    for bad in shared:
        assert forward(**bad) == EINVAL and backward(**bad) == EINVAL, bad
    for bad in (dict(lse=None), dict(dout=None), dict(dout=A + 8), dict(dq=None), dict(dq=A + 4), dict(dkv=None), dict(dkv=A + 8), dict(drope=None),
                dict(drope=A + 8), dict(ws=None), dict(ws=A + 8)):
        assert backward(**bad) == EINVAL, bad
    for bad in (dict(H=129), dict(T=131073), dict(stride=1 << 21), dict(B=2 ** 31 - 1, T=131072)):
        assert forward(**bad) == EUNSUPPORTED and backward(**bad) == EUNSUPPORTED, bad
    assert lib.ngc_latent_replay_workspace_bytes(2, 100, 4, 96) == 0
    assert lib.ngc_latent_replay_workspace_bytes(2, 100, 4, 128) >= 2 * 100 * 4 * (64 + 1) * 4


def test_launches_beyond_the_number_of_threads(lib):
    """2^32 threads and more, and numbers of segments that do not fit, are refused before anything is computed from them."""
    for B, T, H, D in ((100, 131072, 128, 128), (20000, 4096, 128, 64)):
        args = (A, A, A, 64, None, None)
        assert lib.ngc_latent_replay_attn(*args, B, T, H, D, 0.1, A, None, None) == EUNSUPPORTED
        assert lib.ngc_latent_replay_attn_backward(*args, A, A, A, B, T, H, D, 0.1, A, A, A, A, WS, None) == EUNSUPPORTED
    def attn(layer, **kw):
        return lib.ngc_latent_attn(C.byref(latent(Hq=128, **kw)), layer, None, 1024, A, 0.1, 0, A, None, A, WS, None)
    assert attn(0, L=1, B=8192, max_pages=1) == EUNSUPPORTED
    assert attn(-1, L=2, B=2 ** 31 - 1, max_pages=1) == EUNSUPPORTED
    for pc in (cache(L=65535, B=2 ** 31 - 1, Hkv=2, max_pages=1), latent(L=65535, B=300, max_pages=1), cache(L=1, B=2 ** 24, Hkv=1, max_pages=1)):
        assert lib.ngc_paged_extend(C.byref(pc), -1, None, 8, A, A, A, WS, None) == EUNSUPPORTED
    for pc, v in ((cache(L=65535), A), (latent(L=60000), None)):
        assert lib.ngc_paged_fill(C.byref(pc), -1, A, v, None, A, 1 << 24, A, WS, None) == EUNSUPPORTED
