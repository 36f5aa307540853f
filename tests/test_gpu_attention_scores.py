"""GPU: scores that are infinite, in every kernel that forms them (weight 0 for one of
-infinity among others, NaN for a row that has no other, 0 still for a row that sees no key),
and scores so far from 0 that the largest one's product with the scale is not exact."""

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


def _far(torch, dtype, q_len, kv_len, Hq, H, d, seed, size):
    """Queries and keys of which every product and sum is a whole number below 2^24 times
    2^size, so that scores are exact in any order of their sums; a row's largest score belongs
    to one key or to some."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    whole = lambda n, h, top: torch.randint(-top, top + 1, (n, h, d), generator=g,  # noqa: E731
                                            device="cuda").float()
    q = whole(sum(q_len), Hq, 7) * 2.0 ** (size // 2)
    k = whole(sum(kv_len), H, 7) * 2.0 ** (size - size // 2)
    v = torch.randn((sum(kv_len), H, d), generator=g, device="cuda")
    return q.to(t), k.to(t), v.to(t)


def _far_rows(q, k, v, causal):
    """out and lse by the definition, where all but the largest scores' weights are 0."""
    n, Hq, d = q.shape
    t, H = k.shape[:2]
    G = Hq // H
    out, lse, mag = np.zeros((n, Hq, d)), np.zeros((n, Hq)), np.zeros((n, Hq, d))
    for h in range(Hq):
        s = (q[:, h] @ k[:, h // G].T) / math.sqrt(d)
        if causal:
            s = np.where(np.arange(t)[None] <= np.arange(n)[:, None] + t - n, s, -np.inf)
        m = s.max(1, keepdims=True)
        w = (s == m).astype(np.float64)
        lse[:, h] = m[:, 0] + np.log(w.sum(1))
        w /= w.sum(1, keepdims=True)
        out[:, h], mag[:, h] = w @ v[:, h // G], w @ np.abs(v[:, h // G])
    return out, lse, mag


def _check_far(got, lse, want, dtype, t, what, summed=None, rounded=None):
    """Equal weights, whose sum over t keys is rounded in units of `summed` (the mean magnitude
    of what enters it); in bf16 the weights once, relative to `rounded`, and the result.  lse is
    the score: seven roundings of fp32 (the scale, log2(e), their product, that with the score,
    the sum with log2 of the weight, ln(2) and the product with it)."""
    out, want_lse, mag = want
    u, b = 2.0 ** -24, 2.0 ** -8
    summed = mag if summed is None else summed
    bound = (t + 8) * u * summed
    if dtype == "bf16":
        bound = bound + b * (mag if rounded is None else rounded)
    bound = bound + (b if dtype == "bf16" else u) * (np.abs(out) + bound)
    check(got, out, bound, f"out, {what}")
    check(lse, want_lse, 7 * u * np.abs(want_lse) + (t + 8) * u, f"lse, {what}")


@pytest.mark.parametrize("size", [20, 40, 60, 100])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_scores_far_from_zero(torch, shape, dtype, size):
    """Scores of up to 2^(size + 9): differences of 2^size / sqrt(128) at least."""
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len, Hq, H = SHAPES[shape]
    print(f"[gpu-attention-scores] far {shape} {dtype} 2^{size}", flush=True)
    q, k, v = _far(torch, dtype, q_len, kv_len, Hq, H, 128, 4, size)
    out, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    a = c = 0
    for b, (n, t) in enumerate(zip(q_len, kv_len)):
        if b < 4:
            want = _far_rows(f64(q[a:a + n]), f64(k[c:c + t]), f64(v[c:c + t]), True)
            _check_far(f64(out[a:a + n]), f64(lse[a:a + n]), want, dtype, t, f"sequence {b}")
        a, c = a + n, c + t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_ordinary_rows_beside_far_ones(torch, shape, dtype):
    """Rows whose scores are of ordinary size keep their bits, whatever the others' are."""
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len, Hq, H = SHAPES[shape]
    q, k, v = _draw(torch, dtype, q_len, kv_len, Hq, H, 128, 7)
    k = k * 2.0 ** 40
    q[:, ::2] *= 2.0 ** -40
    far = q.clone()
    q[:, 1::2] = 0.0
    ref, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    out, l2 = hf.hf_prompt_attention(far, k, v, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(out[:, ::2], ref[:, ::2]) and torch.equal(l2[:, ::2], lse[:, ::2])
    assert bool(torch.isfinite(out.float()).all()) and bool(torch.isfinite(l2).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("low", [-1e30, -3.3e38], ids=["1e30", "lowest"])
def test_keys_masked_by_their_values(torch, shape, dtype, low):
    """A channel that holds a large negative number in some keys, the first among them (padding
    on the left), takes them out of every row: as if they were not there.  Rows of a causal
    prompt that see only such keys are the mean of these values."""
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len, Hq, H = SHAPES[shape]
    d = 64
    q, k, v = _draw(torch, dtype, q_len, kv_len, Hq, H, d, 5)
    k[..., 5] = 0.0
    q[..., 5] = 1.0
    ends = np.cumsum(kv_len)
    gone = [(np.arange(t) < t // 3) | (np.arange(t) % 11 == 4) for t in kv_len]
    for e, t, x in zip(ends, kv_len, gone):
        k[e - t:e, :, 5][torch.as_tensor(x, device="cuda")] = low
    out, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    a = c = 0
    for b, (n, t) in enumerate(zip(q_len, kv_len)):
        if b < 3:
            kk, vv = f64(k[c:c + t]), f64(v[c:c + t])
            kk[gone[b]] = 0.0
            ref = at.attend(f64(q[a:a + n]), kk, vv, 1 / math.sqrt(d), True, seen=~gone[b])
            bo, bl = bounds(ref, d, t, dtype)
            # rows that see such keys alone: the other channels' products lie below half a step of
            # these scores, which are therefore equal; roundings as in _check_far
            u, h = 2.0 ** -24, 2.0 ** -8 * (dtype == "bf16")
            for i in range(n):
                m = i + t - n + 1
                if gone[b][:m].all():
                    ref["out"][i] = np.repeat(vv[:m].mean(0), Hq // H, 0)
                    mag = np.repeat(np.abs(vv[:m]).mean(0), Hq // H, 0)
                    bo[i] = ((m + 8) * u + h) * mag + max(u, h) * (1 + (m + 8) * u + h) * mag
                    ref["lse"][i] = float(k[c, 0, 5]) / math.sqrt(d) + math.log(m)
                    bl[i] = 7 * u * np.abs(ref["lse"][i]) + (m + 8) * u
            check(f64(out[a:a + n]), ref["out"], bo, f"out of sequence {b}")
            check(f64(lse[a:a + n]), ref["lse"], bl, f"lse of sequence {b}")
        a, c = a + n, c + t


@pytest.mark.parametrize("size", [20, 40, 60, 90])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([3, 1], [70, 200]), ([1], [4001]), ([16], [700])],
                         ids=["whole", "split", "run"])
def test_scores_far_from_zero_over_pages(torch, dtype, size, q_len, kv_len):
    """Keys of whole numbers 0 to 15 times 2^a, which their codes hold exactly; one row of
    ordinary size among the others keeps its bits."""
    from paper_2609_32259_amd import heterofold as hf
    H, Hq, d, P = 2, 6, 128, 32
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(6)
    N = sum(kv_len)
    k = torch.randint(0, 16, (N, H, d), generator=g, device="cuda").float()
    k[:, :, ::32], k[:, :, 1::32] = 0.0, 15.0                # (each group spans 0 to 15)
    k = k * 2.0 ** (size - size // 2)
    v = torch.randint(0, 16, (N, H, d), generator=g, device="cuda").float()
    v[:, :, ::32], v[:, :, 1::32] = 0.0, 15.0
    q = torch.randint(-7, 8, (sum(q_len), Hq, d), generator=g, device="cuda").float() * 2.0 ** (size // 2)
    q[:, 4] = torch.randn((sum(q_len), d), generator=g, device="cuda") * 2.0 ** -(size - size // 2) / 8
    need = [-(-x // P) for x in kv_len]
    table = np.full((len(kv_len), max(need)), -1, np.int32)
    a = 0
    for b, x in enumerate(need):
        table[b, :x] = a + np.arange(x)[::-1]
        a += x
    pages = torch.zeros((1, a, hf.hf_paged_page_bytes(H, d, P)), dtype=torch.uint8, device="cuda")
    cache = hf.PagedKV(pages, torch.as_tensor(table, device="cuda"), H, d, P)
    hf.hf_paged_append(cache, [0] * len(kv_len), kv_len, k, v)
    back = [torch.zeros((N, H, d), device="cuda") for _ in range(2)]
    hf.hf_paged_read(cache, [0] * len(kv_len), kv_len, *back)
    q = q.to(t)
    out, lse = hf.hf_paged_attention(q, cache, q_len, kv_len, return_lse=True)
    alone = q.clone()
    alone[:, [0, 1, 2, 3, 5]] = 0.0
    ref = hf.hf_paged_attention(alone, cache, q_len, kv_len)
    torch.cuda.synchronize()
    assert torch.equal(back[0], k) and torch.equal(back[1], v)
    assert torch.equal(out[:, 4], ref[:, 4])
    heads = [0, 1, 2, 3, 5]
    a = c = 0
    for b, (n, T) in enumerate(zip(q_len, kv_len)):
        want = _far_rows(f64(q[a:a + n]), f64(k[c:c + T]), f64(v[c:c + T]), True)
        # the values' codes (scale 1, offset 0) enter the sums as 16 + code <= 31, the 24 of the
        # operands and the moved offset are taken out, 8 comes from the offsets: 63 at most.
        # Rounded weights count against code - 8
        _check_far(f64(out[a:a + n])[:, heads], f64(lse[a:a + n])[:, heads],
                   tuple(x[:, heads] for x in want), dtype, T, f"sequence {b}", summed=63.0, rounded=8.0)
        a, c = a + n, c + T
