"""Host-side checks of the weights of keys, the eviction and the sampling (no GPU): every call
below fails, or has nothing to do, before the HIP runtime is touched."""

import ctypes as C
from types import SimpleNamespace

import numpy as np
import pytest

from paper_2609_32259_amd import heterofold as hf
from test_attention_host import FAKE, L, _i, _paged, _rows  # noqa: F401

NULL, SHAPE, DTYPE, CAPACITY, UNSUPPORTED = -1, -2, -5, -6, -8


def _w(ptr=FAKE, sb=1000, sl=100, sh=10):
    return hf.hf_key_weights(ptr, sb, sl, sh)


def _weigh(L, q_len=(0,), kv_len=(0,), q=None, k=None, lse=FAKE, scale=0.1, prior=None, decay=1.0,
           w=None, ws=None, wsb=0):
    return L.hf_attention_weights(len(q_len), _i(*q_len), _i(*kv_len), q or _rows(32), k or _rows(),
                                  lse, scale, 1, prior, decay, w or _w(), ws, wsb, None)


def _weigh_paged(L, q_len=(0,), kv_len=(0,), q=None, cache=None, layer=0, lse=FAKE, w=None):
    return L.hf_paged_attention_weights(len(q_len), _i(*q_len), _i(*kv_len), q or _rows(32),
                                        cache or _paged(), layer, lse, 0.1, 1, None, 1.0, w or _w(), None)


def _select(L, kv_len=(0,), keep=(0,), layers=1, H=2, first=0, last=0, w=None, index=FAKE, stride=100):
    return L.hf_evict_select(len(kv_len), layers, H, _i(*kv_len), _i(*keep), first, last, w or _w(),
                             index, stride, None)


def _evict(L, n=(0,), kv_len=(9,), layers=1, index=FAKE, stride=100, k=None, v=None, k_to=None,
           v_to=None, w=None, w_to=None):
    return L.hf_evict_rows(len(n), _i(*n), _i(*kv_len), layers, index, stride, k or _rows(),
                           v or _rows(ptr=2 * FAKE), k_to, v_to, w, w_to, None)


def _evict_paged(L, n=(0,), kv_len=(9,), cache=None, to=None, layer=0, layers=1, index=FAKE,
                 stride=100, w=None, w_to=None):
    return L.hf_paged_evict(len(n), _i(*n), _i(*kv_len), cache or _paged(), to, layer, layers, index,
                            stride, w, w_to, None)


def _sample(L, n=0, vocab=100, dtype=1, x=FAKE, stride=None, T=None, k=None, p=None, m=None, u=FAKE,
            token=FAKE, logprob=None):
    return L.hf_sample_tokens(n, vocab, dtype, x, vocab if stride is None else stride, T, k, p, m, u,
                              token, logprob, None)


def test_nothing_to_do_needs_no_memory(L):  # noqa: F811
    none = _rows(ptr=None)
    assert _weigh(L, q=_rows(32, ptr=None), k=none, lse=None, w=_w(None)) == 0
    assert _weigh(L, (5,), (0,), q=_rows(32, ptr=None), k=none, lse=None, w=_w(None)) == 0
    assert _weigh_paged(L, (5,), (0,), q=_rows(32, ptr=None), lse=None, w=_w(None)) == 0
    assert _select(L, (7,), (0,), w=_w(None), index=None, stride=0) == 0
    assert _evict(L, k=none, v=none, index=None, stride=0) == 0
    assert _evict_paged(L, index=None, stride=0) == 0
    assert _sample(L, x=None, u=None, token=None) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q_len=(-1,)), SHAPE), (dict(kv_len=(-1,)), SHAPE),
    (dict(q_len=(1,), kv_len=(1,), lse=None), NULL),
    (dict(q_len=(1,), kv_len=(1,), lse=FAKE + 2), SHAPE),
    (dict(q_len=(1,), kv_len=(1,), q=_rows(32, ptr=None)), NULL),
    (dict(q_len=(1,), kv_len=(1,), k=_rows(ptr=None)), NULL),
    (dict(q_len=(0,), kv_len=(1,), k=_rows(ptr=None)), NULL),
    (dict(kv_len=(1,), w=_w(None)), NULL), (dict(kv_len=(1,), w=_w(FAKE + 1)), SHAPE),
    (dict(kv_len=(1,), w=_w(sh=-1)), SHAPE), (dict(kv_len=(1,), prior=_w(None)), NULL),
    (dict(kv_len=(1,), prior=_w(), decay=float("nan")), SHAPE),
    (dict(kv_len=(1,), prior=_w(), decay=float("inf")), SHAPE),
    (dict(scale=0.0), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(scale=float("nan")), SHAPE),
    (dict(q=_rows(32, d=64)), SHAPE), (dict(q=_rows(12)), SHAPE),
    (dict(q=_rows(32, dtype=0)), DTYPE), (dict(q=_rows(32, dtype=7)), DTYPE),
    (dict(kv_len=((1 << 30) + 1,)), UNSUPPORTED),
])
def test_weights_refusals(L, kw, status):  # noqa: F811
    assert _weigh(L, **kw) == status, hf.lib().hf_last_error()
    assert hf.lib().hf_last_error()


def test_weights_workspace(L):  # noqa: F811
    size = lambda q, k, Hq=16, H=2, d=128, t=hf.HF_BF16: L.hf_attention_weights_workspace_bytes(  # noqa: E731
        len(q), _i(*q), _i(*k), Hq, H, d, t)
    assert size([1] * 8, [30000] * 8) == 0      # few rows: no parts
    need = size([8192], [8192])                 # few tiles of keys: the rows are cut
    assert need > 0 and need % 256 == 0
    assert size([8192], [8192], Hq=15) == 0 and size([8192], [8192], t=9) == 0 and size([-1], [4]) == 0
    many = dict(q_len=(8192,), kv_len=(8192,), q=_rows(16), k=_rows(2))
    assert _weigh(L, **many) in (0, NULL)       # (NULL, where the causal mask's cut has parts)
    if _weigh_parts(L, many):
        assert _weigh(L, ws=FAKE + 8, wsb=need, **many) == SHAPE
        assert _weigh(L, ws=FAKE, wsb=255, **many) == CAPACITY


def _weigh_parts(L, kw):  # noqa: F811
    return L.hf_attention_weights_workspace_bytes(1, _i(*kw["q_len"]), _i(*kw["kv_len"]), 16, 2, 128,
                                                  hf.HF_BF16) > 0


@pytest.mark.parametrize("kw,status", [
    (dict(layer=2), SHAPE), (dict(cache=_paged(page_tokens=48)), SHAPE),
    (dict(q_len=(1,), kv_len=(257,)), CAPACITY), (dict(q=_rows(32, d=64)), SHAPE),
    (dict(q_len=(1,), kv_len=(1,), cache=_paged(pages=None)), NULL),
    (dict(q_len=(1,), kv_len=(1,), cache=_paged(table=None)), NULL),
    (dict(q_len=(1,), kv_len=(1,), lse=None), NULL), (dict(kv_len=(1,), w=_w(None)), NULL),
])
def test_paged_weights_refusals(L, kw, status):  # noqa: F811
    assert _weigh_paged(L, **kw) in ((status,) if status != CAPACITY else (CAPACITY, SHAPE))
    assert hf.lib().hf_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(kv_len=(-1,)), SHAPE), (dict(keep=(-1,)), SHAPE), (dict(layers=0), SHAPE), (dict(H=0), SHAPE),
    (dict(layers=1 << 20, H=64), SHAPE), (dict(first=-1), SHAPE), (dict(last=-1), SHAPE),
    (dict(kv_len=(9,), keep=(4,), first=3, last=2), SHAPE),
    (dict(kv_len=(9,), keep=(4,), first=2**31 - 1, last=2**31 - 1), SHAPE),
    (dict(kv_len=(9,), keep=(4,), index=None), NULL), (dict(kv_len=(9,), keep=(4,), index=FAKE + 2), SHAPE),
    (dict(kv_len=(9,), keep=(4,), stride=3), CAPACITY), (dict(kv_len=(9,), keep=(4,), w=_w(None)), NULL),
    (dict(kv_len=(9,), keep=(4,), w=_w(sl=-1)), SHAPE), (dict(kv_len=((1 << 30) + 1,)), UNSUPPORTED),
])
def test_choice_refusals(L, kw, status):  # noqa: F811
    assert _select(L, **kw) == status
    assert hf.lib().hf_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(n=(10,)), SHAPE), (dict(n=(-1,)), SHAPE), (dict(layers=0), SHAPE), (dict(layers=70000), SHAPE),
    (dict(n=(4,), index=None), NULL), (dict(n=(4,), index=FAKE + 1), SHAPE), (dict(n=(4,), stride=3), CAPACITY),
    (dict(n=(4,), k=_rows(ptr=None)), NULL), (dict(n=(4,), v=_rows()), SHAPE),
    (dict(v=_rows(dtype=0)), DTYPE), (dict(v=_rows(4)), SHAPE), (dict(v=_rows(d=64)), SHAPE),
    (dict(n=(4,), k_to=_rows(ptr=3 * FAKE)), NULL),
    (dict(n=(4,), k_to=_rows(), v_to=_rows(ptr=3 * FAKE)), SHAPE),
    (dict(n=(4,), k_to=_rows(ptr=3 * FAKE), v_to=_rows(ptr=3 * FAKE)), SHAPE),
    (dict(n=(4,), k_to=_rows(ptr=2 * FAKE), v_to=_rows()), SHAPE),
    (dict(n=(4,), k_to=_rows(4, ptr=3 * FAKE), v_to=_rows(ptr=4 * FAKE)), SHAPE),
    (dict(n=(4,), k_to=_rows(ptr=3 * FAKE), v_to=_rows(ptr=4 * FAKE, dtype=0)), DTYPE),
    (dict(k=_rows(d=8200), v=_rows(d=8200, ptr=2 * FAKE)), UNSUPPORTED),
    (dict(n=(4,), w=_w(None)), NULL), (dict(n=(4,), w_to=_w()), NULL), (dict(n=(4,), w=_w(), w_to=_w()), SHAPE),
    (dict(n=(4,), k_to=_rows(ptr=3 * FAKE), v_to=_rows(ptr=4 * FAKE), w=_w()), NULL),
    (dict(n=(4,), k_to=_rows(ptr=3 * FAKE), v_to=_rows(ptr=4 * FAKE), w=_w(), w_to=_w()), SHAPE),
])
def test_move_refusals(L, kw, status):  # noqa: F811
    assert _evict(L, **kw) == status, hf.lib().hf_last_error()
    assert hf.lib().hf_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(n=(10,)), SHAPE), (dict(layer=1, layers=2), SHAPE), (dict(kv_len=(300,)), CAPACITY),
    (dict(n=(4,), index=None), NULL), (dict(n=(4,), stride=3), CAPACITY),
    (dict(n=(4,), to=_paged()), SHAPE),                                  # the same table
    (dict(n=(4,), to=_paged(table=2 * FAKE, n_pages=11)), SHAPE),        # the same pool, another size
    (dict(n=(4,), to=_paged(table=2 * FAKE, H=4)), SHAPE), (dict(n=(4,), to=_paged(table=2 * FAKE, page_tokens=32)), SHAPE),
    (dict(n=(4,), to=_paged(table=2 * FAKE, d_h=64)), SHAPE),
    (dict(n=(4,), cache=_paged(pages=None)), NULL),
])
def test_paged_move_refusals(L, kw, status):  # noqa: F811
    assert _evict_paged(L, **kw) in ((status,) if status != CAPACITY else (CAPACITY, SHAPE)), hf.lib().hf_last_error()
    assert hf.lib().hf_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), SHAPE), (dict(n=1 << 22), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=(1 << 20) + 1), UNSUPPORTED),
    (dict(dtype=5), DTYPE), (dict(n=1, x=None), NULL), (dict(n=1, u=None), NULL), (dict(n=1, token=None), NULL),
    (dict(n=1, stride=99), SHAPE), (dict(n=1, x=FAKE + 1), SHAPE), (dict(n=1, dtype=0, x=FAKE + 2), SHAPE),
    (dict(n=1, T=FAKE + 1), SHAPE), (dict(n=1, k=FAKE + 2), SHAPE), (dict(n=1, logprob=FAKE + 2), SHAPE),
])
def test_sample_refusals(L, kw, status):  # noqa: F811
    assert _sample(L, **kw) == status, hf.lib().hf_last_error()
    assert hf.lib().hf_last_error()


# The binding: nothing below reaches the library.

torch = pytest.importorskip("torch")


def test_weights_of_the_wrong_kind_are_refused():
    dev = torch.device("cpu")
    for t, error in ((torch.zeros(1, 2, 8, dtype=torch.float64), TypeError), (torch.zeros(1, 2, 7), ValueError),
                     (torch.zeros(1, 3, 8), ValueError), (torch.zeros(2, 8), ValueError),
                     (torch.zeros(1, 2, 16)[:, :, ::2], TypeError)):
        with pytest.raises(error):
            hf._weights(t, (1, 2, 8), "w", dev)
    d = hf._weights(torch.zeros(1, 2, 3, 9), (1, 2, 3, 8), "w", dev)
    assert (d.stride_b, d.stride_l, d.stride_h) == (54, 27, 9)
    with pytest.raises(TypeError):
        hf._own_rows(torch.zeros(1, 1, 8).expand(1, 4, 8), "out")


def test_lists_of_rows_of_the_wrong_kind_are_refused():
    dev = torch.device("cpu")
    for t, error in ((torch.zeros(1, 2, 8), TypeError), (torch.zeros(1, 2, 8, dtype=torch.int64), TypeError),
                     (torch.zeros(1, 8, 2, dtype=torch.int32).transpose(1, 2), TypeError),
                     (torch.zeros(2, 2, 8, dtype=torch.int32), ValueError),
                     (torch.zeros(1, 1, 2, 8, dtype=torch.int32), ValueError)):
        with pytest.raises(error):
            hf._index(t, (1, 2), dev)


def test_weights_that_move_need_a_place():
    dev = torch.device("cpu")
    w = torch.zeros(1, 2, 8)
    args = ((1, 2), [8], [4], dev)
    assert hf._evicted_weights(None, None, *args, False) == (None, None)
    for weights, out, in_place in ((None, w, False), (w, None, False), (w, w.clone(), True),
                                   (torch.zeros(1, 1, 8).expand(1, 2, 8), None, True),
                                   (w, torch.zeros(1, 1, 8).expand(1, 2, 8), False),
                                   (w, torch.zeros(1, 2, 3), False)):
        with pytest.raises((TypeError, ValueError)):
            hf._evicted_weights(weights, out, *args, in_place)


def test_host_tensors_are_refused():
    x = torch.zeros(2, 8)
    rows = torch.zeros(4, 2, 64)
    index = torch.zeros(1, 2, 4, dtype=torch.int32)
    with pytest.raises(TypeError):
        hf.hf_sample_tokens(x, torch.zeros(2))
    with pytest.raises(TypeError):
        hf.hf_sample_tokens(x[0], torch.zeros(2))
    with pytest.raises(TypeError):
        hf.hf_evict_select(torch.zeros(1, 2, 8), [8], [4])
    with pytest.raises(TypeError):
        hf.hf_evict_rows(rows, rows, index, [4], [4])
    with pytest.raises(TypeError):
        hf.hf_attention_weights(rows, rows, torch.zeros(4, 2), [4])
    for t, n, dtype in ((torch.zeros(3), 2, torch.float32), (torch.zeros(2), 2, torch.int32),
                        (torch.zeros(4)[::2], 2, torch.float32)):
        with pytest.raises(TypeError):
            hf._setting(t, n, dtype, "u", torch.device("cpu"))
    cache = SimpleNamespace(batch=1, pages=x, H=2)
    with pytest.raises(ValueError):
        hf.hf_paged_evict(cache, index, [1, 1], [2, 2])
    with pytest.raises(ValueError):
        hf.hf_paged_attention_weights(rows, cache, torch.zeros(4, 2), [1, 1], [2, 2])
    with pytest.raises(ValueError):
        hf.hf_evict_select(torch.zeros(1, 2, 8), np.array([8, 8]), [4])


def test_weights_of_some_layers_only_do_not_shorten_a_paged_cache():
    """(The other layers would have kept their rows, and with them their length.)"""
    from paper_2609_32259_amd.path import evict
    cache = SimpleNamespace(batch=1, pages=torch.zeros(1), L=2, H=2)
    for w in (torch.zeros(1, 2, 8), torch.zeros(1, 1, 2, 8), torch.zeros(1, 2, 3, 8)):
        with pytest.raises(ValueError, match="weights"):
            evict(cache, w, [4], [8])


def test_the_structure_is_the_header_s():
    assert C.sizeof(hf.hf_key_weights) == 32
