"""treewy_hybrid.h: the library exports what it declares, its host checks return the documented codes (no kernel runs), and the
binding names what is wrong."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, M = ctypes.c_void_p(16), ctypes.c_void_p(18)            # aligned and misaligned stand-ins: never dereferenced
OK, INVALID, UNSUPPORTED = 0, 1, 2


@pytest.fixture(scope="module")
def hy():
    from paper_2608_20961_amd import hybrid
    return hybrid


def test_declared_and_exported(hy):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "treewy_hybrid.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(treewy_[a-z_]+)\s*\(", text))
    assert names == set(hy.EXPORTED) and all(hasattr(hy.lib, n) for n in names)


def cache(hy, k=16, v=16, table=16, len_=16, n_pages=4, max_pages=2, page=16):
    return ctypes.byref(hy.Cache(k, v, table, len_, n_pages, max_pages, page))


def rotation(hy, cos=16, sin=16, positions=10, dims=32):
    return ctypes.byref(hy.Rotation(cos, sin, positions, dims))


def test_append_checks(hy):
    def call(k=A, ks=(512, 256, 64), c={}, r={}, path=None, L=4, N=4, B=2, H=2, d=64, dt=1, new=ctypes.c_void_p(32)):
        s = hy.Strides(*ks)
        return hy.lib.treewy_cache_append(k, s, A, s, cache(hy, **c), rotation(hy, **r), path, L, None, N, B, H, d, dt, new, None, None)

    for kw in (dict(N=-1, L=-1), dict(B=-1), dict(L=3), dict(k=None), dict(k=M), dict(ks=(512, 256, 60)), dict(ks=(1 << 62, 256, 64)),
               dict(new=None), dict(new=A), dict(dt=2), dict(c=dict(k=None)), dict(c=dict(len_=None)), dict(c=dict(table=None)),
               dict(c=dict(v=18)), dict(c=dict(page=0)), dict(c=dict(n_pages=-1)), dict(r=dict(cos=None)), dict(r=dict(cos=18)),
               dict(r=dict(positions=0)), dict(r=dict(dims=-16))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(d=96), dict(c=dict(page=12)), dict(c=dict(page=4)), dict(c=dict(page=8192)), dict(r=dict(dims=24)),
               dict(r=dict(dims=80)), dict(path=A, N=257), dict(path=A, L=257), dict(c=dict(max_pages=1 << 30)),
               dict(N=1 << 30, L=1 << 30, B=1 << 10)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(B=0, k=None) == OK


def test_attention_checks(hy):
    def call(q=A, qs=(512, 64, 256), c={}, r={}, shared=0, N=4, B=2, Hq=4, H=2, d=64, dt=1, o=A, ws=A, bytes_=1 << 40):
        s = hy.Strides(*qs)
        return hy.lib.treewy_tree_attention(q, s, A, s, A, s, None, cache(hy, **c), rotation(hy, **r), shared, 0.1, N, B, Hq, H, d, dt,
                                            o, s, ws, bytes_, None, None)

    for kw in (dict(N=-1), dict(Hq=5), dict(H=0), dict(shared=-1), dict(q=None), dict(q=M), dict(o=None), dict(qs=(512, 64, 252)),
               dict(ws=None), dict(ws=M), dict(bytes_=64), dict(dt=3), dict(c=dict(len_=None)), dict(r=dict(sin=None))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(N=257), dict(d=32), dict(c=dict(page=24)), dict(r=dict(dims=8)), dict(B=1 << 24, Hq=1 << 10)):
        assert call(**kw) == UNSUPPORTED, kw
    for kw in (dict(N=0), dict(B=0), dict(Hq=0)):
        assert call(q=None, **kw) == OK, kw


def test_workspace_sizes(hy):
    size = hy.lib.treewy_tree_attention_workspace
    for bad in ((0, 0, 1, 8, 2, 64, 1), (0, 257, 1, 8, 2, 64, 1), (0, 1, 1, 7, 2, 64, 1), (0, 1, 1, 8, 2, 80, 1), (-1, 1, 1, 8, 2, 64, 1)):
        assert size(*bad) == 0
    assert 0 < size(0, 1, 1, 16, 2, 256, 1) < 1 << 28
    assert 0 < size(0, 1, 4096, 64, 8, 128, 1) - 2 * 4096 * 8 * 128 * 2 < 1 << 20      # enough units: nothing is cut, only the draft's rows
    assert size(4096, 1, 64, 32, 8, 128, 1) > 0


def test_sample_checks(hy):
    def call(x=A, u=A, R=2, V=100, dt=1, token=A):
        return hy.lib.treewy_sample(x, V, u, None, None, None, None, R, V, dt, token, None, None, None)

    for kw in (dict(R=-1), dict(V=-1), dict(V=0), dict(dt=2), dict(x=None), dict(u=None), dict(token=None), dict(x=ctypes.c_void_p(17))):
        assert call(**kw) == INVALID, kw
    assert call(V=(1 << 20) + 1) == UNSUPPORTED and call(R=0, x=None) == OK


def test_binding_says_what_is_wrong(hy):
    x, i = torch.zeros(2, 4, 3, 64), torch.zeros(2, dtype=torch.int32)
    assert hy._hybrid.cache_append(x, x, x, x, i, i, *[None] * 7) is None
    assert hy._hybrid.tree_attention(x, x, x, None, x, x, i, i, None, None, 0, 1.0, None, None, None, None) is None
    assert hy._hybrid.sample(x[0, 0], x[0, 0, 0], *[None] * 8) is None
    with pytest.raises(TypeError):
        hy._hybrid.sample(x)
    with pytest.raises(ValueError, match="k must be on a GPU"):
        hy.treewy_cache_append(x, x, x, x, i, i)
    with pytest.raises(TypeError, match="k must be bfloat16 or float32"):
        hy.treewy_cache_append(x.half(), x, x, x, i, i)
    with pytest.raises(ValueError, match="must have 4 dimensions"):
        hy.treewy_tree_attention(x[0], x, x, None, x, x, i, i)
    with pytest.raises(TypeError, match="must be a torch.Tensor"):
        hy.treewy_sample([1.0], x)
    with pytest.raises(ValueError, match="logits must have contiguous rows"):
        hy.treewy_sample(x[0, 0].t(), i)


@pytest.mark.gpu
def test_binding_refusals_on_the_gpu(hy):
    q = torch.zeros(2, 3, 8, 64, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    kv = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16, device="cuda")
    pages = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    table, lens = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    a = dict(q=q, k=kv, v=kv, parent=None, k_pages=pages, v_pages=pages, page_table=table, cache_len=lens)
    call = lambda **kw: hy.treewy_tree_attention(**{**a, **kw})
    ok = call()
    odd = torch.zeros(2, 3, 8, 66, dtype=torch.bfloat16, device="cuda")[..., :64].transpose(1, 2)
    with pytest.raises(ValueError, match="multiples of 16 bytes"):
        call(q=odd)
    with pytest.raises(ValueError, match="multiples of 16 bytes"):
        call(q=torch.zeros(2, 8, 64, 3, dtype=torch.bfloat16, device="cuda").transpose(2, 3))
    with pytest.raises(TypeError, match="v_pages must be"):
        call(v_pages=pages.float())
    with pytest.raises(ValueError, match="page_table must have shape"):
        call(page_table=table[:1])
    with pytest.raises(ValueError, match="cos and sin"):
        call(cos=torch.zeros(4, 8, device="cuda"))
    with pytest.raises(TypeError, match="parent must be"):
        call(parent=torch.zeros(2, 3, dtype=torch.int64, device="cuda"))
    with pytest.raises(hy.TreewyError):
        call(k=torch.zeros(2, 3, 3, 64, dtype=torch.bfloat16, device="cuda"), v=torch.zeros(2, 3, 3, 64, dtype=torch.bfloat16, device="cuda"),
             k_pages=torch.zeros(4, 3, 16, 64, dtype=torch.bfloat16, device="cuda"),
             v_pages=torch.zeros(4, 3, 16, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(hy.TreewyError):
        hy.treewy_cache_append(kv, kv, pages, pages, table, lens, new_len=lens)
    python = type(hy._hybrid)("none")
    for n in ("cache_append", "tree_attention", "sample"):
        setattr(python, n, lambda *x: None)
    native, hy._hybrid = hy._hybrid, python
    try:
        assert torch.equal(ok, call())
    finally:
        hy._hybrid = native


@pytest.mark.gpu
def test_the_native_path_is_loaded(hy):
    assert os.path.basename(hy._hybrid.__file__) == "_hybrid.so"
