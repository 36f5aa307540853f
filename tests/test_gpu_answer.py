"""GPU: a receiver that answers from its cache and keeps it short: attention over the cache, the
weights of its keys, the choice, the move, and the next token, from dense and from paged rows,
eagerly and captured."""

import math

import numpy as np
import pytest

from _attention import bounds, check
from oracle import answer, attention as at
from paper_2609_32259_amd import synth

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


def _path(torch, dtype, d):
    from paper_2609_32259_amd.path import TransferPath
    case = synth.TINY_F32.with_(name="answers", dtype=dtype, batch=2, d_h=d, n_chars=700, L_s=3, L_r=2,
                                H_s=3, H_r=2, rope=(1.0e4, 5.0e5))
    wl = synth.make_workload(case, seed=11, device="cuda")
    path = TransferPath(wl.seg, wl.S, wl.A, wl.bias, wl.rope, case.L_r, case.H_r)
    path.step()
    return case, path


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_shortened_cache_answers_as_its_rows_do(torch, dtype):
    from paper_2609_32259_amd import heterofold as hf
    from paper_2609_32259_amd.path import dense_cache, evict
    d = 128 if dtype == "bf16" else 64
    print(f"[gpu-answer] {dtype}", flush=True)
    case, path = _path(torch, dtype, d)
    B, L, H, Hq = 2, 2, 2, 6
    lens = [int(x) for x in path.r_len]
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(5)
    q_len = [3, 1]
    qs = [torch.randn(4, Hq, d, generator=g).to(t).cuda() for _ in range(L)]
    W = torch.zeros(B, L, H, max(lens), device="cuda")
    for layer, q in enumerate(qs):
        _, lse = path.attend(layer, q, q_len, causal=False, return_lse=True)
        got = path.weigh(layer, q, lse, q_len, causal=False, prior=W[:, layer], decay=0.5, out=W[:, layer])
        assert got.data_ptr() == W[:, layer].data_ptr()
    torch.cuda.synchronize()
    rows = 0
    for b, n in enumerate(q_len):
        # every row's weights sum to 1 (the roundings of the scores, lse and sums: far below 1e-2 in bf16)
        sums = W[b, :, :, :lens[b]].double().sum(-1).cpu().numpy()
        np.testing.assert_allclose(sums, n * Hq / H, rtol=1e-2 if dtype == "bf16" else 1e-5)
        rows += n

    # the same choice for a paged copy and for the dense rows
    keep, first, last = [max(lens) // 3, max(lens) + 1], 2, 5
    P = 32
    need = [-(-x // P) for x in lens]
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    order = torch.randperm(sum(need) + 2, generator=g)
    for b in range(B):
        table[b, :need[b]] = order[sum(need[:b]):sum(need[:b]) + need[b]].int()
    cache = hf.PagedKV(torch.zeros(L, sum(need) + 2, hf.hf_paged_page_bytes(H, d, P), dtype=torch.uint8,
                                   device="cuda"), table.cuda(), H, d, P)
    path.store(cache)
    stored = dense_cache(cache, lens, t, T_cap=max(lens))
    before, weights = path.R.clone(), W.clone()
    paged_w = W.clone()
    n, index = path.evict(W, keep, n_first=first, n_last=last)
    n2, index2 = evict(cache, paged_w, keep, lens, n_first=first, n_last=last)
    torch.cuda.synchronize()
    assert list(n) == [min(a, b) for a, b in zip(keep, lens)] == list(n2)
    short = dense_cache(cache, n, t, T_cap=max(lens))
    for b in range(B):
        m = int(n[b])
        for layer in range(L):
            for h in range(H):
                ids = answer.evict_select(weights[b, layer, h, :lens[b]].cpu().numpy(), keep[b], first, last)
                assert index[b, layer, h, :m].tolist() == ids.tolist() == index2[b, layer, h, :m].tolist()
                at_ = torch.from_numpy(ids).cuda()
                assert torch.equal(path.R[b, layer, :, h, :m], before[b, layer, :, h, at_])
                assert torch.equal(short[b, layer, :, h, :m], stored[b, layer, :, h, at_])
                for w in (W, paged_w):
                    assert torch.equal(w[b, layer, h, :m], weights[b, layer, h, at_])
                    assert torch.equal(w[b, layer, h, m:], weights[b, layer, h, m:])
    assert torch.equal(path.R[:, :, :, :, max(n):], before[:, :, :, :, max(n):])

    # attention over what stayed
    out = path.attend(1, qs[1], q_len, kv_len=n, causal=False)
    torch.cuda.synchronize()
    a = 0
    for b, m in enumerate(q_len):
        k, v = (f64(path.R[b, 1, i, :, :int(n[b])]).transpose(1, 0, 2) for i in range(2))
        ref = at.attend(f64(qs[1][a:a + m]), k, v, 1 / math.sqrt(d), False)
        bo, _ = bounds(ref, d, int(n[b]), dtype)
        check(f64(out[a:a + m]), ref["out"], bo, f"sequence {b}")
        a += m


@pytest.mark.parametrize("paged", [False, True], ids=["dense", "paged"])
def test_a_captured_step_of_answering(torch, paged):
    """Attention, weights, choice, move into another cache, and a token, replayed with other
    queries and random numbers, against the eager calls."""
    from paper_2609_32259_amd import heterofold as hf
    print(f"[gpu-answer] captured paged={paged}", flush=True)
    g = torch.Generator().manual_seed(1)
    B, H, Hq, d, T, P = 2, 2, 8, 64, 200, 32
    kv, keep = [200, 131], [64, 64]
    rnd = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    k, v, q = rnd(B, H, T, d), rnd(B, H, T, d), rnd(B, Hq, d)
    u = torch.rand(B, generator=g).cuda()
    pages = -(-T // P)

    def pool(n):
        return hf.PagedKV(torch.zeros(1, B * n, hf.hf_paged_page_bytes(H, d, P), dtype=torch.uint8, device="cuda"),
                          torch.arange(B * n, dtype=torch.int32, device="cuda").view(B, n), H, d, P)
    cache, to = pool(pages), pool(2)
    hf.hf_paged_append(cache, [0, 0], kv, k, v)
    w, w_to = torch.zeros(B, H, T, device="cuda"), torch.zeros(B, H, 64, device="cuda")
    index = torch.zeros(B, H, 64, dtype=torch.int32, device="cuda")
    k_to = torch.zeros(B, H, 64, d, dtype=torch.bfloat16, device="cuda")
    v_to = torch.zeros_like(k_to)
    top_k = torch.full((B,), 50, dtype=torch.int32, device="cuda")
    top_p = torch.full((B,), 0.9, device="cuda")
    token, logp = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")

    def step():
        if paged:
            out, lse = hf.hf_paged_attention(q, cache, [1, 1], kv, return_lse=True)
            hf.hf_paged_attention_weights(q, cache, lse, [1, 1], kv, out=w)
        else:
            out, lse = hf.hf_prompt_attention(q, k, v, [1, 1], kv, return_lse=True)
            hf.hf_attention_weights(q, k, lse, [1, 1], kv, out=w)
        hf.hf_evict_select(w, kv, keep, 1, 8, out=index)
        if paged:
            hf.hf_paged_evict(cache, index, keep, kv, out=to, weights=w, weights_out=w_to)
        else:
            hf.hf_evict_rows(k, v, index, keep, kv, out=(k_to, v_to), weights=w, weights_out=w_to)
        # (the results stand for the logits that a head would make of them)
        hf.hf_sample_tokens(out.reshape(B, Hq * d), u, top_k=top_k, top_p=top_p, out=token,
                            return_logprob=True, logprob=logp)

    results = lambda: [x.clone() for x in (w, index, w_to, k_to, v_to, to.pages, token, logp)]  # noqa: E731
    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for i in range(4):
        q.copy_(rnd(B, Hq, d))
        u.copy_(torch.rand(B, generator=g))
        step()
        torch.cuda.synchronize()
        eager = results()
        for x in (w, index, w_to, k_to, v_to, to.pages, token, logp):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(results(), eager):
            assert torch.equal(x, y), i
        assert token.min() >= 0 and bool((index[:, :, 1:] > index[:, :, :-1]).all())


def test_offsets_past_32_bits(torch):
    """Rows 2 GiB apart, for every call that takes strides, against the same rows side by side."""
    from paper_2609_32259_amd import heterofold as hf
    print("[gpu-answer] far rows", flush=True)
    g = torch.Generator().manual_seed(2)
    far = torch.empty(9 << 30, dtype=torch.uint8, device="cuda").view(torch.bfloat16)
    T, H, d, step = 4, 2, 64, 1 << 30

    def spread(x, at):  # [1, H, T, d] with tokens `step` elements apart
        y = far.as_strided((1, H, T, d), (0, d, step, 1), at)
        y.copy_(x)
        return y
    x = torch.randn(2, 1, H, T, d, generator=g).bfloat16().cuda()
    k, v = spread(x[0], 0), spread(x[1], 4096)
    for n in (1, 40):  # few and many rows
        q = torch.randn(n, 8, d, generator=g).bfloat16().cuda()
        _, lse = hf.hf_prompt_attention(q, x[0], x[1], [n], [T], causal=False, return_lse=True)
        w = [hf.hf_attention_weights(q, y, lse, [n], [T], causal=False) for y in (k, x[0].contiguous())]
        assert torch.equal(*w)
    index = torch.tensor([[[0, 3], [1, 2]]], dtype=torch.int32, device="cuda")
    hf.hf_evict_rows(k, v, index, [2], [T])
    hf.hf_evict_rows(x[0], x[1], index, [2], [T])
    for y, z in ((k, x[0]), (v, x[1])):
        assert torch.equal(y, z)

    w = far.view(torch.float32).as_strided((2, 1, 50), (step, 50, 1), 8192)
    w.copy_(torch.rand(2, 1, 50, generator=g))
    ids = hf.hf_evict_select(w, [50, 50], [20, 20])
    for b in range(2):
        assert ids[b, 0].tolist() == answer.evict_select(w[b, 0].cpu().numpy(), 20).tolist()

    logits = far.as_strided((4, 1000), (step, 1), 65536)
    logits.copy_(torch.randn(4, 1000, generator=g).bfloat16())
    u = torch.rand(4, generator=g).cuda()
    assert torch.equal(hf.hf_sample_tokens(logits, u), hf.hf_sample_tokens(logits.contiguous(), u))
