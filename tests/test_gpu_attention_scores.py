"""GPU: scores that are infinite, in every kernel that forms them: weight 0 for one of
-infinity among others, NaN for a row that has no other, 0 still for a row that sees no key."""

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


# q_len, kv_len, H_q, H: by keys; by keys and split; by rows (256 tiles at least); rows and split
SHAPES = {
    "few": ([9, 2], [80, 300], 6, 3),
    "split": ([1, 2], [5001, 700], 4, 1),
    "many": ([70, 33] * 32, [70, 90] * 32, 16, 8),
    "suffix": ([300], [3100], 16, 4),
}


def _draw(torch, dtype, q_len, kv_len, Hq, H, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rnd = lambda n, h: torch.randn((n, h, d), generator=g, device="cuda").to(t)  # noqa: E731
    return rnd(sum(q_len), Hq), rnd(sum(kv_len), H), rnd(sum(kv_len), H)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_scores_of_minus_infinity(torch, shape, dtype, d):
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len, Hq, H = SHAPES[shape]
    print(f"[gpu-attention-scores] -inf {shape} {dtype} d={d}", flush=True)
    q, k, v = _draw(torch, dtype, q_len, kv_len, Hq, H, d, 1)
    q[..., 5] = 1.0
    ends = np.cumsum(kv_len)
    # of each sequence: the first 60% of the keys of head 0 (with them whole parts of a cut
    # range), all of the last head's; the other heads (if any) are left alone
    gone = [np.arange(t) < (6 * t) // 10 for t in kv_len]
    for e, t, g in zip(ends, kv_len, gone):
        if H > 1:
            k[e - t:e, H - 1, 5] = -math.inf
        k[e - t:e, 0, 5][torch.as_tensor(g, device="cuda")] = -math.inf
    out, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, causal=False, return_lse=True)
    torch.cuda.synchronize()
    G = Hq // H
    if H > 1:
        assert bool(torch.isnan(out[:, Hq - G:].float()).all())
        assert bool((lse[:, Hq - G:] == -math.inf).all())
    a = c = 0
    for b, (n, t) in enumerate(zip(q_len, kv_len)):
        if b < 3:
            heads = 1 if H > 1 else H
            kk = f64(k[c:c + t, :heads])
            kk[gone[b]] = 0.0
            ref = at.attend(f64(q[a:a + n, :G]), kk, f64(v[c:c + t, :heads]), 1 / math.sqrt(d), False,
                            seen=~gone[b])
            bo, bl = bounds(ref, d, t, dtype)
            check(f64(out[a:a + n, :G]), ref["out"], bo, f"out of sequence {b}")
            check(f64(lse[a:a + n, :G]), ref["lse"], bl, f"lse of sequence {b}")
        a, c = a + n, c + t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_infinite_queries(torch, shape, dtype):
    """Whatever the sign of the keys against it: a row with an infinite query is NaN, also the
    first of a causal prompt, which sees one key."""
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len, Hq, H = SHAPES[shape]
    q, k, v = _draw(torch, dtype, q_len, kv_len, Hq, H, 128, 2)
    ref = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
    q2 = q.clone()
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    for i in range(0, q.shape[0], 7):
        hit[i, i % Hq] = True
        q2[i, i % Hq, i % 128] = math.inf if i % 2 else -math.inf
    out = hf.hf_prompt_attention(q2, k, v, q_len, kv_len)
    torch.cuda.synchronize()
    assert bool(torch.isnan(out[hit].float()).all())
    assert torch.equal(out[~hit], ref[~hit])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [70, 4001], ids=["whole", "split"])
def test_infinite_queries_over_pages(torch, dtype, T):
    """NaN where a row sees a key, 0 where all its pages are holes."""
    from paper_2609_32259_amd import heterofold as hf
    H, Hq, d, P = 2, 6, 128, 32
    n = -(-T // P)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(3)
    pages = torch.zeros((1, n, hf.hf_paged_page_bytes(H, d, P)), dtype=torch.uint8, device="cuda")
    table = torch.stack([torch.arange(n, dtype=torch.int32), torch.full((n,), -1, dtype=torch.int32),
                         torch.full((n,), -1, dtype=torch.int32)]).cuda()
    table[2, n // 2] = n // 2                  # one page among holes
    cache = hf.PagedKV(pages, table, H, d, P)
    k, v = (torch.randn((T, H, d), generator=g, device="cuda") for _ in range(2))
    one = hf.PagedKV(pages, table[:1].contiguous(), H, d, P)
    hf.hf_paged_append(one, [0], [T], k, v)
    q = torch.randn((6, Hq, d), generator=g, device="cuda").to(t)
    ref = hf.hf_paged_attention(q, cache, [2, 2, 2], [T, T, T])
    q[::2, 1, 3] = math.inf
    q[::2, 4, 70] = -math.inf
    out, lse = hf.hf_paged_attention(q, cache, [2, 2, 2], [T, T, T], return_lse=True)
    torch.cuda.synchronize()
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    hit[::2, 1] = hit[::2, 4] = True
    hit[2:4] = False
    assert bool(torch.isnan(out[hit].float()).all())
    assert torch.equal(out[~hit], ref[~hit])
    assert bool((out[2:4] == 0).all()) and bool((lse[2:4] == -math.inf).all())
