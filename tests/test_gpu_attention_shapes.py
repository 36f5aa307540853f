"""GPU: attention in the shapes that large batches take (tiles of rows that fill the chip),
wide groups, shared heads, queries that are not finite, batches with empty sequences, pools
past 4 GiB, graphs that share a workspace."""

import math

import numpy as np
import pytest

from _attention import bounds, check
from oracle import attention as at

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU test needs a GPU"
    from paper_2609_32259_amd import heterofold
    heterofold.lib()
    return torch


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _draw(torch, dtype, q_len, kv_len, Hq, H, d, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rnd = lambda n, h: torch.randn((n, h, d), generator=g).to(t).cuda()  # noqa: E731
    return 1.5 * rnd(sum(q_len), Hq), rnd(sum(kv_len), H), rnd(sum(kv_len), H)


def _compare(q, k, v, out, lse, q_len, kv_len, dtype, causal, some=None):
    d, a, c = q.shape[2], 0, 0
    for b, (n, t) in enumerate(zip(q_len, kv_len)):
        if n and (some is None or b in some):
            ref = at.attend(f64(q[a:a + n]), f64(k[c:c + t]), f64(v[c:c + t]), 1 / math.sqrt(d), causal)
            bo, bl = bounds(ref, d, t, dtype)
            check(f64(out[a:a + n]), ref["out"], bo, f"out of sequence {b}")
            check(f64(lse[a:a + n]), ref["lse"], bl, f"lse of sequence {b}")
        a, c = a + n, c + t


def _many(seed, top):
    """64 sequences, some without queries, some without keys, some with fewer keys than
    queries; with 4 heads their tiles of rows fill the chip."""
    rng = np.random.default_rng(seed)
    q_len = rng.integers(0, top, size=64)
    kv_len = q_len + rng.integers(0, 120, size=64)
    q_len[[3, 62]] = 0
    kv_len[[5, 63]] = 0
    q_len[5], q_len[7], kv_len[7] = 2, 40, 33
    q_len[q_len == 0] += (np.arange(64)[q_len == 0] != 3) & (np.arange(64)[q_len == 0] != 62)
    return [int(x) for x in q_len], [int(x) for x in kv_len]


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,G", [(128, 1), (64, 3)])
def test_many_sequences(torch, d, G, dtype, causal):
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len = _many(1, 60)
    print(f"[gpu-attention-shapes] many {dtype} d={d} G={G} causal={causal}", flush=True)
    q, k, v = _draw(torch, dtype, q_len, kv_len, 6 * G, 6, d, 2)
    out, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, causal=causal, return_lse=True)
    torch.cuda.synchronize()
    _compare(q, k, v, out, lse, q_len, kv_len, dtype, causal)


@pytest.mark.parametrize("dtype,q_len,kv_len", [
    ("bf16", [620], [620]), ("bf16", [300], [3100]), ("bf16", [33, 290], [2100, 2777]),
    ("f32", [401], [401]), ("f32", [150], [2500]),
], ids=["prompt", "split", "split ragged", "fp32 prompt", "fp32 split"])
def test_long_tiles_of_rows(torch, dtype, q_len, kv_len):
    from paper_2609_32259_amd import heterofold as hf
    print(f"[gpu-attention-shapes] long {dtype} {q_len} {kv_len}", flush=True)
    q, k, v = _draw(torch, dtype, q_len, kv_len, 32, 8, 128, 3)
    out, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    # (the oracle on one group of heads: rows of every tile and part)
    for h in (0, 7):
        _compare(q[:, 4 * h:4 * h + 2], k[:, h:h + 1], v[:, h:h + 1], out[:, 4 * h:4 * h + 2],
                 lse[:, 4 * h:4 * h + 2], q_len, kv_len, dtype, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_seen_has_no_influence(torch, dtype):
    """The batch above with one key or value that is not finite: the rows that do not see it
    keep their bits, and so do all other sequences."""
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len = _many(4, 60)
    H = 6
    q, k, v = _draw(torch, dtype, q_len, kv_len, 2 * H, H, 128, 5)
    ref, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    b = max(range(64), key=lambda i: q_len[i])
    n, t = q_len[b], kv_len[b]
    q0, k0 = sum(q_len[:b]), sum(kv_len[:b])
    for what, bad in (("v", math.nan), ("v", math.inf), ("v", -math.inf), ("k", math.nan), ("k", math.inf)):
        for row in (1, n // 2, n - 1):
            k2, v2 = k.clone(), v.clone()
            (v2 if what == "v" else k2)[k0 + t - n + row, 1, 5] = bad
            out, l2 = hf.hf_prompt_attention(q, k2, v2, q_len, kv_len, return_lse=True)
            torch.cuda.synchronize()
            hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
            hit[q0 + row:q0 + n, 2:4, 5 if what == "v" else slice(None)] = True
            assert torch.equal(out[~hit], ref[~hit]), (what, bad, row)
            if bad != bad:
                assert bool(torch.isnan(out[hit].float()).all())
            elif what == "v":
                assert bool((out[hit].float() == bad).all())
            if what == "v":
                assert torch.equal(l2, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("many", [False, True], ids=["few", "many"])
def test_queries_that_are_not_finite(torch, dtype, many):
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len = _many(6, 60) if many else ([9, 2], [80, 300])
    q, k, v = _draw(torch, dtype, q_len, kv_len, 12, 6, 128, 7)
    ref = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
    q2 = q.clone()
    q2[2, 3, 9] = math.nan
    q2[4, 0, 1] = math.inf
    out = hf.hf_prompt_attention(q2, k, v, q_len, kv_len)
    torch.cuda.synchronize()
    hit = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
    hit[2, 3] = hit[4, 0] = True
    assert torch.equal(out[~hit], ref[~hit])
    assert bool(torch.isnan(out[hit].float()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,H", [(71, 1), (64, 1), (33, 3)])
def test_wide_groups_and_shared_heads(torch, dtype, Hq, H):
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len = [3, 1, 5], [70, 200, 5]
    print(f"[gpu-attention-shapes] wide {dtype} {Hq}/{H}", flush=True)
    q, k, v = _draw(torch, dtype, q_len, kv_len, Hq, H, 64, 8)
    out, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    _compare(q, k, v, out, lse, q_len, kv_len, dtype, True)
    if H == 1:   # the same rows named as one head for each query head (stride 0)
        wide = hf.hf_prompt_attention(q, k.expand(-1, Hq, -1), v.expand(-1, Hq, -1), q_len, kv_len)
        torch.cuda.synchronize()
        _compare(q, k, v, wide, lse, q_len, kv_len, dtype, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged_batch_of_many(torch, dtype):
    """64 paged sequences, empty ones among them, against dense attention in fp32 over the
    rows read back."""
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len = _many(9, 9)
    H, Hq, d, P = 3, 12, 128, 32
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v = _draw(torch, dtype, q_len, kv_len, Hq, H, d, 10)
    need = [-(-x // P) for x in kv_len]
    order = np.random.default_rng(11).permutation(sum(need))
    table = np.full((64, max(need)), -1, np.int32)
    a = 0
    for b, x in enumerate(need):
        table[b, :x] = order[a:a + x]
        a += x
    pages = torch.zeros((1, a, hf.hf_paged_page_bytes(H, d, P)), dtype=torch.uint8, device="cuda")
    cache = hf.PagedKV(pages, torch.as_tensor(table, device="cuda"), H, d, P)
    hf.hf_paged_append(cache, [0] * 64, kv_len, k, v)
    back = [torch.zeros((sum(kv_len), H, d), device="cuda") for _ in range(2)]
    hf.hf_paged_read(cache, [0] * 64, kv_len, *back)
    out, lse = hf.hf_paged_attention(q, cache, q_len, kv_len, return_lse=True)
    want, lse2 = hf.hf_prompt_attention(q.float(), *back, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    empty = torch.isinf(lse2)
    assert torch.equal(torch.isinf(lse), empty) and bool((out.float()[empty] == 0).all())
    # scores are off by (d + 4) a + 4 half steps of fp32 with a = scale sum |q_e k_e| < 60
    # (|q| < 1.5 x 5, |k| < 5 over 128 channels of mean 0.64): under 2^-11, on either side; the
    # weights by twice that, 2^-9 of the largest value in all.  In bf16 a weight times its
    # group's scale and the result besides: two half steps
    lim = float(back[1].abs().max()) * (2.0 ** -9 + (2 * 2.0 ** -8 if dtype == "bf16" else 0))
    assert float((out.float() - want).abs().max()) <= lim
    assert float((lse - lse2)[~empty].abs().max()) <= 2.0 ** -10 + 1e-5


def test_pool_past_four_gigabytes(torch):
    from paper_2609_32259_amd import heterofold as hf
    H, Hq, d, P, T = 8, 32, 128, 64, 500
    n = (5 << 30) // hf.hf_paged_page_bytes(H, d, P)
    pages = torch.empty((1, n, hf.hf_paged_page_bytes(H, d, P)), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v, q = (torch.randn((m, h, d), generator=g, device="cuda").bfloat16()
               for m, h in ((T, H), (T, H), (2, Hq)))
    outs = []
    for ids in (np.arange(8), n - 1 - np.arange(8)):
        cache = hf.PagedKV(pages, torch.as_tensor(ids[None].astype(np.int32), device="cuda"), H, d, P)
        hf.hf_paged_append(cache, [0], [T], k, v)
        back = [torch.zeros((T, H, d), device="cuda") for _ in range(2)]
        hf.hf_paged_read(cache, [0], [T], *back)
        outs.append((hf.hf_paged_attention(q, cache, [2], [T]), *back))
    torch.cuda.synchronize()
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert float((outs[0][1] - k.float()).abs().max()) < float(k.float().abs().max())


def test_two_graphs_of_one_workspace(torch):
    """Replayed one after another, with eager work between, each gives the eager result."""
    from paper_2609_32259_amd import heterofold as hf
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    sets = []
    for i, T in enumerate((9000, 5000)):
        q, k, v = _draw(torch, "bf16", [1], [T], 8, 2, 128, 12 + i)
        run = lambda q=q, k=k, v=v, T=T: hf.hf_prompt_attention(q, k, v, [1], [T], workspace=ws)  # noqa: E731
        ref = run().clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        sets.append((graph, out, ref, run))
    for _ in range(3):
        for graph, out, ref, run in sets:
            out.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref)
            assert torch.equal(run(), ref)
