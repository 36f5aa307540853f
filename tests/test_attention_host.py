"""Host-side checks of the attention and paged-cache calls (no GPU): every call below
fails, or has nothing to do, before the HIP runtime is touched."""

import ctypes as C
import os

import numpy as np
import pytest

from paper_2609_32259_amd import heterofold as hf

NULL, SHAPE, DTYPE, CAPACITY, UNSUPPORTED = -1, -2, -5, -6, -8
FAKE = 0x10000


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(hf.LIB_PATH):
        from paper_2609_32259_amd import build
        build.build()
    return hf.lib()


def _i(*v):
    return (C.c_int32 * len(v))(*v)


def _rows(H=8, d=128, dtype=1, ptr=FAKE, sb=-1, sl=0, sh=None, st=None):
    return hf.hf_rows(ptr, dtype, H, d, sb, sl, d if sh is None else sh, H * d if st is None else st)


def _prompt(L, B=1, q_len=(0,), kv_len=(0,), q=None, k=None, v=None, out=None, scale=0.1, lse=None,
            ws=None, wsb=0):
    q = _rows(32) if q is None else q
    return L.hf_prompt_attention(B, _i(*q_len), _i(*kv_len), q, k or _rows(), v or _rows(),
                                 out or q, scale, 1, lse, ws, wsb, None)


def _paged(**kw):
    a = dict(pages=FAKE, table=FAKE, table_stride=4, n_pages=10, L=2, H=8, d_h=128, page_tokens=64)
    a.update(kw)
    return hf.hf_paged_kv(*a.values())


def _attend(L, cache=None, q=None, layer=0, q_len=(0,), kv_len=(0,), scale=0.1):
    q = _rows(32) if q is None else q
    return L.hf_paged_attention(len(q_len), _i(*q_len), _i(*kv_len), q, cache or _paged(), layer, q,
                                scale, 1, None, None, 0, None)


def _append(L, cache=None, start=(0,), n=(0,), layer=0, layers=1, k=None, v=None, theta=0.0,
            pos0=None):
    return L.hf_paged_append(len(n), _i(*start), _i(*n), cache or _paged(), layer, layers,
                             k or _rows(), v or _rows(), theta, pos0, None)


def test_nothing_to_do_needs_no_memory(L):
    empty = _rows(32, ptr=None)
    none = _rows(ptr=None)
    assert _prompt(L, q=empty, k=none, v=none) == 0
    assert _prompt(L, q=empty, k=none, v=none, q_len=(0,), kv_len=(7,)) == 0
    assert _attend(L, q=empty, kv_len=(300,)) == 0   # (no query row: the table is not read)
    assert _append(L, k=none, v=none) == 0
    assert L.hf_paged_read(1, _i(0), _i(0), _paged(), 0, 2, none, none, None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), SHAPE), (dict(B=65), SHAPE), (dict(q_len=(-1,)), SHAPE), (dict(kv_len=(-1,)), SHAPE),
    (dict(q_len=(1,), q=_rows(32, ptr=None)), NULL),
    (dict(q_len=(1,), kv_len=(1,), k=_rows(ptr=None)), NULL),
    (dict(q_len=(1,), kv_len=(1,), v=_rows(ptr=None)), NULL),
    (dict(q=_rows(32, ptr=FAKE + 8)), SHAPE), (dict(k=_rows(ptr=FAKE + 2)), SHAPE),
    (dict(q=_rows(30)), SHAPE), (dict(q=_rows(32, dtype=7)), DTYPE), (dict(k=_rows(dtype=3)), DTYPE),
    (dict(k=_rows(dtype=0), v=_rows(dtype=0)), DTYPE), (dict(k=_rows(dtype=0)), DTYPE),
    (dict(out=_rows(32, dtype=0)), DTYPE), (dict(out=_rows(16)), SHAPE),
    (dict(k=_rows(d=64), v=_rows(d=64)), SHAPE), (dict(v=_rows(4)), SHAPE),
    (dict(q=_rows(32, d=96), k=_rows(d=96), v=_rows(d=96)), UNSUPPORTED),
    (dict(k=_rows(st=1028)), SHAPE), (dict(v=_rows(sh=-128)), SHAPE), (dict(k=_rows(sb=-2)), SHAPE),
    (dict(k=_rows(sb=12)), SHAPE), (dict(out=_rows(32, st=64)), SHAPE), (dict(out=_rows(32, sh=64)), SHAPE),
    (dict(k=_rows(st=(1 << 23) + 8)), UNSUPPORTED),
    (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE),
    (dict(scale=3e38), SHAPE), (dict(lse=FAKE + 1), SHAPE),
    (dict(q_len=(1,), kv_len=((1 << 30) + 1,)), UNSUPPORTED),
    (dict(q_len=((1 << 31) - 1,), kv_len=(5,)), SHAPE),
    (dict(q_len=(1,), kv_len=(40000,)), NULL),                          # a split range needs a workspace
    (dict(q_len=(1,), kv_len=(40000,), ws=FAKE + 128, wsb=1 << 30), SHAPE),
    (dict(q_len=(1,), kv_len=(40000,), ws=FAKE, wsb=100), CAPACITY),
])
def test_prompt_attention_refuses(L, kw, status):
    assert _prompt(L, **kw) == status
    assert L.hf_last_error().decode()


@pytest.mark.parametrize("kw,status", [
    (dict(pages=None), NULL), (dict(table=None), NULL), (dict(pages=FAKE + 4), SHAPE),
    (dict(table=FAKE + 2), SHAPE), (dict(table_stride=-1), SHAPE), (dict(n_pages=0), SHAPE),
    (dict(L=0), SHAPE), (dict(H=0), SHAPE), (dict(d_h=96), UNSUPPORTED), (dict(page_tokens=48), SHAPE),
    (dict(page_tokens=16), SHAPE), (dict(page_tokens=512), SHAPE), (dict(H=16), SHAPE), (dict(d_h=64), SHAPE),
])
def test_paged_calls_refuse_caches(L, kw, status):
    cache = _paged(**kw)
    # (q of 32 heads on 16 is a valid grouping: that one is the rows' mismatch)
    if kw != dict(H=16):
        assert _attend(L, cache) == status
    assert _append(L, cache) == status
    assert L.hf_paged_read(1, _i(0), _i(0), cache, 0, 1, _rows(), _rows(), None) == status


def test_paged_calls_refuse(L):
    for layer, layers in ((-1, 1), (2, 1), (1, 2), (0, 0), (0, 1 << 30)):
        assert _append(L, layer=layer, layers=layers) == SHAPE
    assert _attend(L, layer=2) == SHAPE and _attend(L, layer=-1) == SHAPE
    assert _attend(L, q=_rows(30)) == SHAPE
    assert _attend(L, q=_rows(32, d=64)) == SHAPE
    assert _attend(L, q_len=(1,), kv_len=(257,)) == CAPACITY     # four pages of 64
    assert _append(L, start=(200,), n=(57,)) == CAPACITY
    assert _append(L, start=(-1,), n=(1,)) == SHAPE
    assert _append(L, n=(-1,)) == SHAPE
    assert _append(L, n=(1,), k=_rows(ptr=None)) == NULL
    assert _append(L, n=(1,), v=_rows(ptr=None)) == NULL
    assert _append(L, k=_rows(dtype=0)) == DTYPE
    assert _append(L, k=_rows(4)) == SHAPE
    assert _append(L, k=_rows(sl=4)) == SHAPE
    for theta in (-1.0, float("inf"), float("nan")):
        assert _append(L, theta=theta) == SHAPE
    assert _append(L, pos0=_i(-1)) == SHAPE
    assert _append(L, n=(1,), pos0=_i((1 << 31) - 2)) == SHAPE
    assert L.hf_paged_read(1, _i(0), _i(0), _paged(), 0, 1, _rows(st=64), _rows(), None) == SHAPE
    assert L.hf_paged_append(1, _i(0), None, _paged(), 0, 1, _rows(), _rows(), 0.0, None, None) == NULL


def test_sizes(L):
    assert hf.hf_paged_page_bytes(8, 128, 64) == 8 * 64 * 160
    assert hf.hf_paged_page_bytes(2, 64, 32) == 2 * 32 * 80
    for bad in ((0, 128, 64), (8, 96, 64), (8, 128, 48), (8, 128, 0)):
        assert hf.hf_paged_page_bytes(*bad) == 0
    f = hf.hf_attention_workspace_bytes
    assert f([1], [40000], 32, 8, 128, hf.HF_BF16) > 0
    assert f([1], [40000], 32, 8, 128, hf.HF_BF16, paged=True) > 0
    assert f([8192], [8192], 32, 8, 128, hf.HF_BF16) == 0        # the rows fill the chip
    assert f([1], [5], 32, 8, 128, hf.HF_BF16) == 0
    for bad in (([1], [1], 30, 8, 128, 1), ([1], [1], 32, 8, 96, 1), ([1], [1], 32, 8, 128, 5),
                ([-1], [1], 32, 8, 128, 1)):
        assert f(*bad) == 0


def test_workspaces_are_those_of_the_plan(L):
    """Random lengths: with the bytes that a call asks for it passes the workspace check,
    causal or not (and is refused for its row stride, which is looked at after that); with
    less it does not, causal or not."""
    rng = np.random.default_rng(0)
    far = _rows(st=(1 << 23) + 8)
    cut = 0
    for _ in range(200):
        B = int(rng.integers(1, 9))
        q_len = [int(x) for x in rng.integers(1, [2, 40, 3000][int(rng.integers(3))], size=B)]
        kv = [int(x) for x in rng.integers(0, [50, 3000, 100000][int(rng.integers(3))], size=B)]
        need = hf.hf_attention_workspace_bytes(q_len, kv, 32, 8, 128, hf.HF_BF16)
        call = lambda ws, n, causal: L.hf_prompt_attention(  # noqa: E731
            B, _i(*q_len), _i(*kv), _rows(32), far, far, _rows(32), 0.1, causal, None, ws, n, None)
        for causal in (0, 1):
            assert call(FAKE, need, causal) == UNSUPPORTED
        if need:
            cut += 1
            assert CAPACITY in [call(FAKE, need - 256, causal) for causal in (0, 1)]
            assert SHAPE in [call(FAKE + 128, need, causal) for causal in (0, 1)]
            assert NULL in [call(None, 0, causal) for causal in (0, 1)]
    assert 20 < cut < 180


def test_binding_refuses(L):
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        hf.hf_prompt_attention(x, x, x, [4])                     # not on a GPU
    with pytest.raises(TypeError):
        hf.PagedKV(torch.zeros((1, 2, 8 * 64 * 160), dtype=torch.uint8),
                   torch.zeros((1, 2), dtype=torch.int32), 8, 128)
    with pytest.raises(ValueError):
        hf.PagedKV(x, x, 8, 100)
    with pytest.raises(ValueError):
        hf._lens([[1, 2]], "n") if isinstance([[1, 2]][0], int) else hf._lens(np.zeros((2, 2), np.int32), "n")
    with pytest.raises(ValueError):
        hf._lens([1, 2], "n", 3)
    with pytest.raises(ValueError):
        hf._lens([1 << 31], "n")
    cpu = torch.device("cpu")
    for t, lens, layers in ((x, [5], None), (x[None], [1, 2], None), (x[None], [9], None), (x[0], [1], None),
                            (x.transpose(0, 2), [4], None), (x[None, None], [1], 2)):
        with pytest.raises((TypeError, ValueError)):
            hf._head_rows(t, lens, "t", cpu, layers)
    r = hf._head_rows(x[None, None], [8], "t", cpu, 1)           # [B, L, H, T, d]
    assert (r.H, r.d_h, r.stride_t, r.stride_h) == (4, 128, 128, 1024)
