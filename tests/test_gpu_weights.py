"""Attention weights of keys on the GPU against the fp64 definition.

Bounds.  u is half a step of fp32 (2^-24).  A score is a sum of d products, of magnitude
`arg`: (d + 4) arg u with the scale and the exponent's fused multiply-add; the base-2 exponent
holds lse with three half steps (its product with log2 e, and the constant's and the sum's own
rounding), and the exponential adds four.  The sum of a key's weights over n rows adds at most
n / 16 + 24 half steps (halves within 16 rows, one after another over tiles, then lanes and
waves), decay and prior two.  Over pages the codes enter as 16 + code, so that a score is
formed from terms of up to 47 s + |o| a channel instead of s code + o.
"""

import math

import numpy as np
import pytest

from oracle import answer as ans
from oracle import attention as att

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU test needs a GPU"
    from paper_2609_32259_amd import heterofold
    heterofold.lib()
    return torch


def _f64(t):
    return t.double().cpu().numpy()


def _lse(q, k, scale, causal, seen=None):
    """fp32 log-sum-exps of one sequence in fp64, rounded."""
    n, Hq, _ = q.shape
    t, H = k.shape[0], k.shape[1]
    out = np.full((n, Hq), -np.inf, np.float32)
    for i in range(n):
        ok = np.ones(t, bool) if seen is None else seen.copy()
        if causal:
            ok &= np.arange(t) <= i + t - n
        for h in range(Hq if ok.any() else 0):
            s = scale * (k[ok, h // (Hq // H)] @ q[i, h])
            m = s.max()
            out[i, h] = m + np.log(np.exp(s - m).sum())
    return out


def _check(got, ref, d, rows, what, prior=None, decay=1.0):
    w = ref["w"]
    mag = np.abs(w) + (0 if prior is None else 2 * abs(decay) * np.abs(prior))
    bound = U * ((d + 4) * ref["err"] + (rows / 16 + 24 + 4) * mag) + 1e-37
    assert np.array_equal(np.isnan(got), np.isnan(w)), f"{what}: NaN elsewhere"
    off = np.abs(got - w)
    fine = ~np.isnan(w)
    assert (off[fine] <= bound[fine]).all(), f"{what}: worst {(off[fine] / bound[fine]).max():.2f} of the bound"


def _dense(torch, dtype, q_len, kv_len, Hq, H, d, causal, packed, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = (spread * torch.randn((sum(q_len) + 2, Hq, d), generator=g)).to(t)
    if packed:
        k = torch.randn((sum(kv_len) + 3, H, d), generator=g).to(t)
        at = np.concatenate([[0], np.cumsum(kv_len)])
        keys = [k[int(at[b]):int(at[b]) + n] for b, n in enumerate(kv_len)]
    else:
        k = torch.randn((len(kv_len), 3, H, max(max(kv_len), 1) + 5, d), generator=g).to(t)[:, 1]
        keys = [k[b, :, :n].transpose(0, 1) for b, n in enumerate(kv_len)]
    scale = 1.0 / math.sqrt(d)
    row, lse, per = 0, [], []
    for b, n in enumerate(q_len):
        x, y = _f64(q[row:row + n]), _f64(keys[b])
        l = _lse(x, y, scale, causal)
        lse.append(l)
        per.append((x, y, l))
        row += n
    dev = k.cuda() if packed else torch.stack([k]).cuda()[0]
    return q.cuda(), dev, torch.as_tensor(np.concatenate(lse)).cuda().contiguous(), per, scale


CASES = [
    # dtype, q_len, kv_len, Hq, H, d, causal, packed
    ("bf16", [1], [1], 4, 4, 128, True, True),
    ("bf16", [1, 0, 1], [7, 5, 0], 8, 2, 128, True, False),
    ("bf16", [1, 1], [200, 333], 28, 4, 128, True, False),
    ("bf16", [33, 1, 64], [33, 1, 64], 6, 2, 64, True, True),
    ("bf16", [5, 40], [3, 17], 3, 1, 128, True, False),      # rows that see nothing
    ("bf16", [70, 90], [65, 129], 8, 8, 64, False, False),
    ("bf16", [257], [257], 4, 1, 128, True, True),           # eight waves share the rows
    ("bf16", [300, 2], [130, 600], 7, 1, 64, True, False),
    ("f32", [1, 3], [1, 40], 8, 2, 64, True, False),
    ("f32", [33, 20], [33, 77], 5, 1, 128, True, False),
    ("f32", [0, 290], [10, 290], 2, 2, 64, True, True),
    ("f32", [12], [100], 4, 2, 128, False, False),
]


@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]} q{c[1]} k{c[2]} {c[3]}/{c[4]}x{c[5]}" for c in CASES])
@pytest.mark.parametrize("with_prior", [False, True], ids=["new", "prior"])
def test_dense(torch, case, with_prior):
    from paper_2609_32259_amd import heterofold as hf
    dtype, q_len, kv_len, Hq, H, d, causal, packed = case
    q, k, lse, per, scale = _dense(torch, dtype, q_len, kv_len, Hq, H, d, causal, packed, 3, 1.5)
    T = max(kv_len)
    out = torch.full((len(kv_len), H, T + 4), 7.5, device="cuda")
    prior = torch.rand((len(kv_len), H, T + 1), device="cuda") if with_prior else None
    got = hf.hf_attention_weights(q, k, lse, q_len, kv_len, causal=causal, prior=prior, decay=0.5, out=out)
    assert got is out
    for b, (x, y, l) in enumerate(per):
        n = kv_len[b]
        pr = _f64(prior[b, :, :n]) if with_prior else None
        ref = ans.key_weights(x, y, l, scale, causal, prior=pr, decay=0.5)
        _check(_f64(out[b, :, :n]), ref, d, q_len[b] * Hq // H, f"sequence {b}", pr, 0.5)
        assert (out[b, :, n:] == 7.5).all(), "numbers behind the keys were written"


def test_many_keys_in_wide_tiles(torch):
    """Enough keys and rows for tiles of 128 keys, against the sums of torch in fp64."""
    from paper_2609_32259_amd import heterofold as hf
    g = torch.Generator(device="cuda").manual_seed(5)
    n, T, Hq, H, d = 300, 16500, 4, 2, 128
    q = torch.randn((n, Hq, d), generator=g, device="cuda").bfloat16()
    k = torch.randn((1, H, T, d), generator=g, device="cuda").bfloat16()
    s = torch.matmul(q.double().transpose(0, 1), k[0].double().repeat_interleave(2, 0).transpose(1, 2).contiguous())
    s = s / math.sqrt(d)
    hide = torch.arange(T, device="cuda") > torch.arange(n, device="cuda")[:, None] + T - n
    s = s.masked_fill(hide, -math.inf)
    lse = torch.logsumexp(s, -1).t().float().contiguous()
    w = torch.exp(s - lse.t().double()[..., None]).view(H, 2, n, T).sum((1, 2))
    got = hf.hf_attention_weights(q, k, lse, [n], [T])[0].double()
    # arg: scale sum |q k| < scale |q| |k| < 1.2 sqrt(d) * 1.5 for these rows, and lse < 11
    bound = U * ((d + 4) * 21 + 3 * 11 + 2 * n / 16 + 28) * w
    assert ((got - w).abs() <= bound).all(), float(((got - w).abs() / bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_a_row_does_not_see_has_no_influence(torch, dtype):
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len, Hq, H, d = [40, 3], [40, 100], 4, 2, 64
    q, k, lse, per, scale = _dense(torch, dtype, q_len, kv_len, Hq, H, d, True, False, 9)
    want = hf.hf_attention_weights(q, k, lse, q_len, kv_len)
    k2, q2 = k.clone(), q.clone()
    k2[0, :, 40:] = math.nan                   # rows behind the keys
    k2[1, :, 100:] = math.inf
    q2[43:] = math.nan                         # rows behind the queries
    got = hf.hf_attention_weights(q2, k2, lse, q_len, kv_len)
    assert torch.equal(got, want)
    k2[0, 1, 25] = math.nan                    # a key that the rows from 25 on see
    got = hf.hf_attention_weights(q2, k2, lse, q_len, kv_len)
    bad = torch.isnan(got)
    assert bad[0, 1, 25] and bad.sum() == 1
    assert torch.equal(torch.where(bad, 0.0, got), torch.where(bad, 0.0, want))


def test_rows_of_infinite_scores_and_far_ones(torch):
    from paper_2609_32259_amd import heterofold as hf
    d = 64
    q = torch.zeros((3, 1, d), device="cuda")
    k = torch.zeros((1, 1, 40, d), device="cuda")
    q[:, 0, 0] = torch.tensor([1.0, 1e30, -1.0], device="cuda")
    k[0, 0, :, 0] = -math.inf                   # row 0: all scores -inf; row 2: all +inf
    lse = torch.tensor([[-math.inf], [-math.inf], [0.0]], device="cuda")
    w = hf.hf_attention_weights(q[:2], k, lse[:2], [2], [40], causal=False)
    assert torch.isnan(w).all()                 # 0/0, as the result of such a row
    # scores of 2^39: lse's own rounding decides the largest one's weight, which is at most 1;
    # all others have 0
    q = torch.zeros((2, 1, d), device="cuda")
    q[:, 0, 0] = 2.0 ** 20
    k = torch.zeros((1, 1, 40, d), device="cuda")
    k[0, 0, :, 0] = torch.arange(40, device="cuda") * 2.0 ** 17
    s = 2.0 ** 20 * 39 * 2.0 ** 17 / 8
    w = hf.hf_attention_weights(q, k, torch.full((2, 1), s, device="cuda"), [2], [40], causal=False)
    assert (w[0, 0, :39] == 0).all() and 0 <= w[0, 0, 39] <= 2.0
    # lse past every score: nothing
    w = hf.hf_attention_weights(q, k, torch.full((2, 1), math.inf, device="cuda"), [2], [40], causal=False)
    assert (w == 0).all()


def _cache(torch, H, d, P, kv_len, seed, holes=()):
    from paper_2609_32259_amd import heterofold as hf
    rng = np.random.default_rng(seed)
    pages_of = [-(-n // P) for n in kv_len]
    n_pages = sum(pages_of) + 2
    ids = rng.permutation(n_pages)
    table = np.full((len(kv_len), max(max(pages_of), 1)), -1, np.int32)
    pool = rng.integers(0, 256, (n_pages, att.page_bytes(H, d, P)), dtype=np.uint8)
    keys, at = [], 0
    for b, n in enumerate(pages_of):
        rows = rng.standard_normal((2, max(n, 1) * P, H, d)).astype(np.float32)
        c, s, o = att.quantise(rows)
        for j in range(n):
            p = int(ids[at])
            sl = slice(j * P, j * P + P)
            pool[p] = att.pack_page(c[:, sl], s[:, sl], o[:, sl], H, d, P)
            table[b, j] = -1 if (b, j) in holes else p
            at += 1
        keys.append((att.dequantise(c[0], s[0], o[0]), s[0], o[0]))
    cache = hf.PagedKV(torch.as_tensor(pool)[None].cuda(), torch.as_tensor(table).cuda(), H, d, P)
    return cache, keys


PAGED = [
    ("bf16", [1], [1], 4, 4, 128, 32, ()),
    ("bf16", [1, 1, 1], [70, 0, 300], 20, 4, 128, 64, ()),
    ("bf16", [3, 0, 17], [65, 40, 257], 6, 2, 64, 32, ((2, 1),)),
    ("bf16", [40], [40], 8, 1, 128, 128, ()),
    ("f32", [1, 2], [33, 100], 8, 2, 128, 32, ((1, 0),)),
    ("f32", [20], [300], 3, 1, 64, 256, ()),
]


@pytest.mark.parametrize("case", PAGED, ids=[f"{c[0]} q{c[1]} k{c[2]} {c[3]}/{c[4]}x{c[5]}" for c in PAGED])
def test_paged(torch, case):
    from paper_2609_32259_amd import heterofold as hf
    dtype, q_len, kv_len, Hq, H, d, P, holes = case
    cache, keys = _cache(torch, H, d, P, kv_len, 11, holes)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.randn((sum(q_len), Hq, d), generator=torch.Generator().manual_seed(1)).to(t)
    scale = 1.0 / math.sqrt(d)
    row, lse, refs = 0, [], []
    prior = torch.rand((len(kv_len), H, max(kv_len)))
    for b, n in enumerate(q_len):
        x, (y, s, o) = _f64(q[row:row + n]), keys[b]
        m = kv_len[b]
        seen = np.array([(b, j // P) not in holes for j in range(m)], bool)
        l = _lse(x, y[:m], scale, True, seen)
        lse.append(l)
        r = ans.key_weights(x, y[:m], l, scale, True, seen, _f64(prior[b, :, :m]), 0.9)
        # the magnitudes that the codes' form goes through: 47 s + |o| a channel
        wide = np.repeat(47.0 * s + np.abs(o), 32, axis=-1)[:m].astype(np.float64)
        new = dict(w=r["w"], err=np.zeros_like(r["err"]))
        for i in range(n):
            for h in range(Hq):
                ok = seen & (np.arange(m) <= i + m - n)
                x0 = np.where(ok, np.exp(np.where(ok, scale * (y[:m, h // (Hq // H)] @ x[i, h]), 0) - (l[i, h] if ok.any() else 0)), 0)
                new["err"][h // (Hq // H)] += x0 * (scale * (wide[:, h // (Hq // H)] @ np.abs(x[i, h])) +
                                                   (3 * abs(l[i, h]) / d if ok.any() else 0))
        refs.append(new)
        row += n
    lse = torch.as_tensor(np.concatenate(lse)).cuda().contiguous()
    out = prior.cuda()
    hf.hf_paged_attention_weights(q.cuda(), cache, lse, q_len, kv_len, prior=out, decay=0.9, out=out)
    for b, r in enumerate(refs):
        m = kv_len[b]
        _check(_f64(out[b, :, :m]), r, d + 12, q_len[b] * Hq // H, f"sequence {b}", _f64(prior[b, :, :m]), 0.9)
        assert torch.equal(out[b, :, m:].cpu(), prior[b, :, m:])


def test_paged_words_that_are_not_finite_stay_with_their_tokens(torch):
    from paper_2609_32259_amd import heterofold as hf
    H, d, P, n = 2, 128, 32, 90
    cache, _ = _cache(torch, H, d, P, [n], 4)
    q = torch.randn((2, 4, d), generator=torch.Generator().manual_seed(2)).cuda().bfloat16()
    lse = torch.full((2, 4), 5.0, device="cuda")
    want = hf.hf_paged_attention_weights(q, cache, lse, [2], [n])
    pages = cache.pages.clone()
    view = pages.view(-1, H, att.page_bytes(1, d, P))
    page = int(cache.table[0, 1])
    at = P * d + 10 * d // 8                     # words of token 32 + 10's keys, head 1
    view[page, 1, at:at + 4] = 255               # NaN, NaN
    page = int(cache.table[0, 2])
    view[page, :, P * d + 26 * d // 8:P * d + 27 * d // 8] = 255  # token 90: behind the keys
    got = hf.hf_paged_attention_weights(q, hf.PagedKV(pages, cache.table, H, d, P), lse, [2], [n])
    bad = torch.isnan(got)
    assert bad[0, 1, 42] and bad.sum() == 1
    assert torch.equal(torch.where(bad, 0.0, got), torch.where(bad, 0.0, want))


@pytest.mark.parametrize("paged", [False, True], ids=["dense", "paged"])
def test_weights_of_the_attention_sum_to_its_rows(torch, paged):
    """As a decoding step uses them: attention, then the weights by its lse; every row's
    weights sum to 1."""
    from paper_2609_32259_amd import heterofold as hf
    H, Hq, d, P = 2, 10, 128, 64
    kv = [500, 131]
    q = torch.randn((4, Hq, d), generator=torch.Generator().manual_seed(8)).cuda().bfloat16()
    if paged:
        cache, _ = _cache(torch, H, d, P, kv, 21)
        _, lse = hf.hf_paged_attention(q, cache, [3, 1], kv, return_lse=True)
        w = hf.hf_paged_attention_weights(q, cache, lse, [3, 1], kv)
    else:
        k = torch.randn((2, H, 500, d), generator=torch.Generator().manual_seed(7)).cuda().bfloat16()
        _, lse = hf.hf_prompt_attention(q, k, k, [3, 1], kv, return_lse=True)
        w = hf.hf_attention_weights(q, k, lse, [3, 1], kv)
    rows = torch.tensor([3.0, 1.0], device="cuda")[:, None] * Hq / H
    # the lse is good to a few 1e-6, the weights likewise
    assert ((w.double().sum(-1) - rows).abs() < 2e-5 * rows).all()


def test_streams_and_graphs(torch):
    from paper_2609_32259_amd import heterofold as hf
    q, k, lse, _, _ = _dense(torch, "bf16", [1, 1], [200, 300], 8, 2, 128, True, False, 2)
    want = hf.hf_attention_weights(q, k, lse, [1, 1], [200, 300])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = hf.hf_attention_weights(q, k, lse, [1, 1], [200, 300], stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hf.hf_attention_weights(q, k, lse, [1, 1], [200, 300], prior=out, decay=1.0, out=out)
    total = torch.zeros_like(want)
    for i in range(4):
        q.mul_(0.9)
        graph.replay()
        total = hf.hf_attention_weights(q, k, lse, [1, 1], [200, 300], prior=total)
        torch.cuda.synchronize()
        assert torch.equal(out, total), f"replay {i}"


@pytest.mark.parametrize("dtype,d,q", [("bf16", 128, 1), ("bf16", 64, 37), ("f32", 64, 3), ("f32", 128, 36)])
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_a_large_paged_batch_is_its_sequences(torch, dtype, d, q, causal):
    """Enough tokens that a workgroup has several tiles, of fewer than 65 query rows a head and of
    more: the same bits as each sequence in a call of its own (one tile a workgroup), which the
    definition is held against above.  (A key's sum goes by its rows, in the same order.)"""
    from paper_2609_32259_amd import heterofold as hf
    B, H, Hq, P, T = 48, 8, 16, 32, 700
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    print(f"[gpu-weights] large paged batch {dtype} d={d} q={q} causal={causal}", flush=True)
    g = torch.Generator().manual_seed(d + q)
    kv_len = [(T - 13 * b if b % 5 else b) for b in range(B)]
    pages = -(-T // P)
    order = torch.randperm(B * pages, generator=g).int().view(B, pages)
    order[3, 2] = -1
    cache = hf.PagedKV(torch.zeros(1, B * pages, hf.hf_paged_page_bytes(H, d, P), dtype=torch.uint8, device="cuda"),
                       order.cuda(), H, d, P)
    x = torch.randn(B, H, T, d, generator=g).to(t).cuda()
    hf.hf_paged_append(cache, [0] * B, kv_len, x, x)
    qs = torch.randn(B * q, Hq, d, generator=g).to(t).cuda()
    _, lse = hf.hf_paged_attention(qs, cache, [q] * B, kv_len, causal=causal, return_lse=True)
    out = torch.full((B, H, T), 7.0, device="cuda")
    hf.hf_paged_attention_weights(qs, cache, lse, [q] * B, kv_len, causal=causal, out=out)
    for b in range(B):
        one = hf.PagedKV(cache.pages, cache.table[b:b + 1], H, d, P)
        w = torch.full((1, H, T), 7.0, device="cuda")
        hf.hf_paged_attention_weights(qs[b * q:(b + 1) * q], one, lse[b * q:(b + 1) * q], [q], kv_len[b:b + 1],
                                      causal=causal, out=w)
        assert torch.equal(out[b], w[0]), b
        assert bool((w[0, :, kv_len[b]:] == 7.0).all())
