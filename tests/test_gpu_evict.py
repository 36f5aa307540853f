"""The choice of the tokens that stay, and their rows moved together: whole numbers and
bits, so that everything is compared exactly."""

import numpy as np
import pytest

from oracle import answer as ans
from oracle import attention as att

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU test needs a GPU"
    from paper_2609_32259_amd import heterofold
    heterofold.lib()
    return torch


def _values(rng, kind, shape):
    x = rng.standard_normal(shape).astype(np.float32)
    if kind == "ties":
        x = np.round(x * 2) / 2                       # a few values, zeros of both signs among them
        x[rng.random(shape) < 0.1] = -0.0
    elif kind == "equal":
        x[:] = 0.25
    elif kind == "odd":
        x = np.exp(3 * x)
        u = rng.random(shape)
        x[u < 0.05] = np.nan
        x[(u > 0.05) & (u < 0.1)] = np.inf
        x[(u > 0.1) & (u < 0.15)] = -np.inf
        x[(u > 0.15) & (u < 0.2)] = 1e-42
    elif kind == "near":                              # neighbours: the last bits decide
        x = (np.float32(1.0).view(np.uint32) + rng.integers(0, 9000, shape).astype(np.uint32)).view(np.float32)
    return x


@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "odd", "near"])
@pytest.mark.parametrize("T,keep,first,last", [
    (1, 1, 0, 0), (1, 0, 0, 0), (2, 1, 0, 1), (64, 63, 0, 0), (65, 20, 4, 16), (300, 5, 2, 3), (300, 299, 0, 0),
    (1000, 400, 4, 100), (8192, 4096, 4, 32), (8193, 100, 0, 1), (20001, 15000, 7, 0), (32768, 1, 0, 0),
    (32769, 9000, 4, 64), (100000, 50000, 0, 0)])
def test_choice(torch, kind, T, keep, first, last):
    from paper_2609_32259_amd import heterofold as hf
    rng = np.random.default_rng(T)
    H = 2
    x = _values(rng, kind, (1, H, T + 3))
    w = torch.as_tensor(x).cuda()
    out = torch.full((1, H, keep + 2), -7, dtype=torch.int32, device="cuda")
    hf.hf_evict_select(w, [T], [keep], first, last, out=out)
    got = out.cpu().numpy()
    assert (got[:, :, min(keep, T):] == -7).all()
    for h in range(H):
        assert np.array_equal(got[0, h, :keep], ans.evict_select(x[0, h, :T], keep, first, last)), h


def test_choice_in_batches(torch):
    """Layers, ragged lengths, sequences that keep all or nothing, a view of longer rows."""
    from paper_2609_32259_amd import heterofold as hf
    rng = np.random.default_rng(1)
    B, L, H, T = 4, 3, 2, 700
    x = _values(rng, "ties", (B, L + 1, H, T + 9))
    w = torch.as_tensor(x).cuda()[:, 1:, :, 5:5 + T]
    kv, keep = [700, 0, 65, 333], [100, 9, 70, 0]
    keep[3] = 200
    out = hf.hf_evict_select(w, kv, keep, 3, 10)
    assert out.shape == (B, L, H, 200) and out.dtype == torch.int32
    got = out.cpu().numpy()
    for b in range(B):
        n = min(kv[b], keep[b])
        for l in range(L):
            for h in range(H):
                want = ans.evict_select(x[b, l + 1, h, 5:5 + kv[b]], keep[b], 3, 10) if kv[b] else np.zeros(0)
                assert np.array_equal(got[b, l, h, :n], want), (b, l, h)


def _rising(rng, kv, n, lead):
    """[B, *lead, max n] rising numbers, and the most for numpy."""
    out = np.full((len(kv),) + lead + (max(max(n), 1),), 99, np.int32)
    for b in range(len(kv)):
        for at in np.ndindex(lead):
            out[(b,) + at][:n[b]] = np.sort(rng.permutation(kv[b])[:n[b]])
    return out


DENSE = [("bf16", 128, [50, 0, 7], [200, 30, 7]), ("f32", 64, [3, 130], [500, 131]), ("f32", 128, [1], [1]),
         ("bf16", 64, [200, 256], [256, 256]), ("bf16", 40, [33], [90]), ("f32", 512, [70], [300])]


@pytest.mark.parametrize("in_place", [False, True], ids=["other", "in place"])
@pytest.mark.parametrize("case", DENSE, ids=str)
def test_dense_rows(torch, case, in_place):
    from paper_2609_32259_amd import heterofold as hf
    dtype, d, n, kv = case
    rng = np.random.default_rng(3)
    B, L, H = len(n), 2, 3
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    R = torch.randn((B, L + 1, 2, H, max(kv) + 6, d), generator=torch.Generator().manual_seed(1)).to(t)
    w0 = torch.rand((B, L, H, max(kv) + 2), generator=torch.Generator().manual_seed(2))
    index = _rising(rng, kv, n, (L, H))
    if n[0] > 3:
        index[0, :, :, :3] = [0, 1, 2]                # a front that stays
        index[0, :, :, 3:n[0]] = np.sort(3 + np.argsort(rng.random((L, H, kv[0] - 3)))[..., :n[0] - 3], -1)
    dev, w = R.cuda(), w0.cuda()
    k, v = dev[:, 1:, 0], dev[:, 1:, 1]
    if in_place:
        got = hf.hf_evict_rows(k, v, torch.as_tensor(index).cuda(), n, kv, weights=w)
        new_w, old, old_w = w, R[:, 1:], w0
        got = torch.stack([got[0], got[1]], 2)
    else:
        to = torch.full((2, B, L, H, max(n) + 3, d), 4.0, dtype=t, device="cuda")
        new_w = torch.full((B, L, H, max(n) + 1), 4.0, device="cuda")
        hf.hf_evict_rows(k, v, torch.as_tensor(index).cuda(), n, kv, out=(to[0], to[1]), weights=w, weights_out=new_w)
        got = torch.stack([to[0], to[1]], 2)
        old = torch.full(got.shape, 4.0).to(t)
        old_w = torch.full(new_w.shape, 4.0)
        assert torch.equal(dev.cpu(), R) and torch.equal(w.cpu(), w0)
    got, new_w = got.cpu(), new_w.cpu()
    for b in range(B):
        for l in range(L):
            for h in range(H):
                at = torch.as_tensor(index[b, l, h, :n[b]]).long()
                for role in range(2):
                    assert torch.equal(got[b, l, role, h, :n[b]], R[b, 1 + l, role, h][at]), (b, l, role, h)
                    assert torch.equal(got[b, l, role, h, n[b]:], old[b, l, role, h, n[b]:])
                assert torch.equal(new_w[b, l, h, :n[b]], w0[b, l, h][at])
                assert torch.equal(new_w[b, l, h, n[b]:], old_w[b, l, h, n[b]:])
    if in_place:
        assert torch.equal(dev[:, 0].cpu(), R[:, 0])


@pytest.mark.parametrize("in_place", [False, True], ids=["other", "in place"])
def test_packed_rows(torch, in_place):
    """Sequences back to back: in place each stays where it begins, elsewhere they close up."""
    from paper_2609_32259_amd import heterofold as hf
    rng = np.random.default_rng(5)
    n, kv, H, d = [4, 0, 90], [9, 5, 100], 2, 64
    x = torch.randn((2, sum(kv) + 2, H, d), generator=torch.Generator().manual_seed(1))
    index = _rising(rng, kv, n, (H,))
    dev = x.cuda()
    if in_place:
        hf.hf_evict_rows(dev[0], dev[1], torch.as_tensor(index).cuda(), n, kv)
        got, start = dev.cpu(), [0, 9, 14]
    else:
        to = torch.zeros((2, sum(n), H, d), device="cuda")
        hf.hf_evict_rows(dev[0], dev[1], torch.as_tensor(index).cuda(), n, kv, out=(to[0], to[1]))
        got, start = to.cpu(), [0, 4, 4]
    for b, at in enumerate([0, 9, 14]):
        for h in range(H):
            rows = torch.as_tensor(index[b, h, :n[b]]).long() + at
            for role in range(2):
                assert torch.equal(got[role, start[b]:start[b] + n[b], h], x[role][rows, h])
                if in_place:
                    assert torch.equal(got[role, at + n[b]:at + kv[b], h], x[role][at + n[b]:at + kv[b], h])


def test_numbers_outside_are_clamped(torch):
    from paper_2609_32259_amd import heterofold as hf
    x = torch.randn((2, 1, 1, 20, 64), device="cuda")
    index = torch.tensor([[[-5, 3, 3, 1 << 30]]], dtype=torch.int32, device="cuda")
    to = torch.zeros((2, 1, 1, 4, 64), device="cuda")
    hf.hf_evict_rows(x[0], x[1], index, [4], [20], out=(to[0], to[1]))
    assert torch.equal(to, x[:, :, :, [0, 3, 3, 19]])


def _pool(rng, H, d, P, pages):
    c = rng.integers(0, 16, (pages, 2, P, H, d))
    s = np.exp(rng.standard_normal((pages, 2, P, H, d // 32))).astype(np.float32)
    s = (s.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
    o = rng.standard_normal(s.shape).astype(np.float32)
    o = (o.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
    return c, s, o


PAGED = [(128, 32, [40, 33, 0], [100, 60, 20]), (128, 64, [31], [64]), (64, 32, [64, 1], [65, 33]),
         (64, 128, [200], [300]), (128, 256, [255, 300], [256, 500])]


@pytest.mark.parametrize("in_place", [False, True], ids=["other", "in place"])
@pytest.mark.parametrize("case", PAGED, ids=str)
def test_paged_rows(torch, case, in_place):
    from paper_2609_32259_amd import heterofold as hf
    d, P, n, kv = case
    rng = np.random.default_rng(d + P)
    B, L, H = len(n), 3, 2
    need = [-(-t // P) for t in kv]
    pages = sum(need) * 2 + 2
    c, s, o = _pool(rng, H, d, P, L * pages)
    raw = np.stack([att.pack_page(c[p], s[p], o[p], H, d, P) for p in range(L * pages)]).reshape(L, pages, -1)
    ids = rng.permutation(pages)
    table, other = (np.full((B, max(need) + 1), -1, np.int32) for _ in range(2))
    at = 0
    for b in range(B):
        table[b, :need[b]] = ids[at:at + need[b]]
        other[b, :need[b]] = ids[at + need[b]:at + 2 * need[b]]
        at += 2 * need[b]
    pool = torch.as_tensor(raw).cuda()
    cache = hf.PagedKV(pool, torch.as_tensor(table).cuda(), H, d, P)
    to = None if in_place else hf.PagedKV(pool, torch.as_tensor(other).cuda(), H, d, P)
    layer, layers = 1, 2
    index = _rising(rng, kv, n, (layers, H))
    w0 = torch.rand((B, layers, H, max(kv)))
    w, w_to = w0.cuda(), torch.zeros((B, layers, H, max(max(n), 1)), device="cuda")
    got = hf.hf_paged_evict(cache, torch.as_tensor(index).cuda(), n, kv, out=to, layer=layer, weights=w,
                            weights_out=None if in_place else w_to)
    assert got is (cache if in_place else to)
    after = pool.cpu().numpy()
    want = raw.copy()
    dst = table if in_place else other
    new_w = w if in_place else w_to
    fields = lambda l, p: (x.reshape(L, pages, *x.shape[1:])[l, p] for x in (c, s, o))  # noqa: E731
    for l in range(layers):
        edit = {}
        for b in range(B):
            for i in range(n[b]):
                p = int(dst[b, i // P])
                if p not in edit:
                    edit[p] = [x.copy() for x in fields(layer + l, p)]
                for h in range(H):
                    t = int(index[b, l, h, i])
                    src = list(fields(layer + l, int(table[b, t // P])))
                    for e, f in zip(edit[p], src):
                        e[:, i % P, h] = f[:, t % P, h]
            for h in range(H):
                rows = torch.as_tensor(index[b, l, h, :n[b]]).long()
                assert torch.equal(new_w[b, l, h, :n[b]].cpu(), w0[b, l, h][rows])
        for p, e in edit.items():
            want[layer + l, p] = att.pack_page(*e, H, d, P)
    assert np.array_equal(after, want)


def test_holes_of_the_pages(torch):
    """A token out of a hole is 0, one into a hole is dropped; nothing else moves."""
    from paper_2609_32259_amd import heterofold as hf
    d, P, H = 64, 32, 1
    rng = np.random.default_rng(2)
    c, s, o = _pool(rng, H, d, P, 6)
    raw = np.stack([att.pack_page(c[p], s[p], o[p], H, d, P) for p in range(6)])[None]
    pool = torch.as_tensor(raw).cuda()
    cache = hf.PagedKV(pool, torch.tensor([[0, -1, 1]], dtype=torch.int32).cuda(), H, d, P)
    to = hf.PagedKV(pool, torch.tensor([[3, 77]], dtype=torch.int32).cuda(), H, d, P)
    index = torch.tensor([[[3, 40, 70] + list(range(71, 91)) + list(range(0, 17))]], dtype=torch.int32).cuda()
    hf.hf_paged_evict(cache, index, [40], [96], out=to)
    got = pool.cpu().numpy()[0]
    gc, gs, go = att.unpack_page(got[3], H, d, P)
    for i, t in enumerate(index[0, 0, :32].tolist()):
        p = [0, None, 1][t // P]
        for a, b in ((gc, c), (gs, s), (go, o)):
            want = np.zeros_like(a[:, i]) if p is None else b[p][:, t % P]
            assert np.array_equal(a[:, i], want), i
    for p in (0, 1, 2, 4, 5):
        assert np.array_equal(got[p], raw[0, p])


def test_graph_of_choice_and_move(torch):
    from paper_2609_32259_amd import heterofold as hf
    B, L, H, T, d = 2, 2, 2, 300, 64
    R = torch.randn((B, L, 2, H, T, d), device="cuda")
    w = torch.rand((B, L, H, T), device="cuda")
    to = torch.zeros((2, B, L, H, 100, d), device="cuda")
    w_to = torch.zeros((B, L, H, 100), device="cuda")
    n, kv = [100, 90], [300, 200]
    index = torch.zeros((B, L, H, 100), dtype=torch.int32, device="cuda")

    def step():
        hf.hf_evict_select(w, kv, n, 4, 10, out=index)
        hf.hf_evict_rows(R[:, :, 0], R[:, :, 1], index, n, kv, out=(to[0], to[1]), weights=w, weights_out=w_to)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        w.copy_(torch.rand_like(w))
        graph.replay()
        got = to.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, to)
        at = index[1, 1, 1, :90].long()
        assert torch.equal(to[0, 1, 1, 1, :90], R[1, 1, 0, 1][at])


def test_choice_of_many_rows_is_that_of_few(torch):
    """(More rows than are worked on at once take fewer waves each.)"""
    from paper_2609_32259_amd import heterofold as hf
    print("[gpu-evict] many rows", flush=True)
    rng = np.random.default_rng(9)
    w = rng.standard_normal((2, 300, 1500)).astype(np.float32)
    w[:, ::3] = np.round(w[:, ::3], 1)   # ties
    w[:, ::7, ::5] = np.nan
    t = torch.from_numpy(w).cuda()
    kv, keep = [1500, 1111], [700, 300]
    many = torch.full((2, 300, 700), -5, dtype=torch.int32, device="cuda")
    few = many.clone()
    hf.hf_evict_select(t, kv, keep, 3, 4, out=many)
    for b in range(2):
        part = few[b:b + 1]
        hf.hf_evict_select(t[b:b + 1], kv[b:b + 1], keep[b:b + 1], 3, 4, out=part)
    assert torch.equal(many, few)
    for b, h in ((0, 0), (0, 7), (1, 21), (1, 299)):
        want = ans.evict_select(w[b, h, :kv[b]], keep[b], 3, 4)
        assert many[b, h, :keep[b]].tolist() == want.tolist()
    assert bool((many[1, :, 300:] == -5).all())
