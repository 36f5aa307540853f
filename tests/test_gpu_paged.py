"""GPU: the paged cache held in 4 bits.  Appended pages against the oracle's codes, bit
for bit; rows read back; attention over pages against the fp64 oracle on the values that
the codes stand for, within the bounds of ``_attention``; holes, shared pages, rows that
see nothing, what lies in masked places; a run of all of it together."""

import math

import numpy as np
import pytest

from _attention import U32, UB, bounds, check, logical
from oracle import attention as at
from oracle import rope as ro

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


def _cache(torch, tokens, L, H, d, P, seed, extra=2):
    """A pool of arbitrary bytes and a table in random page order."""
    from paper_2609_32259_amd import heterofold as hf
    rng = np.random.default_rng(seed)
    need = [-(-t // P) for t in tokens]
    n = sum(need) + extra
    pages = torch.as_tensor(rng.integers(0, 256, size=(L, n, at.page_bytes(H, d, P)), dtype=np.uint8),
                            device="cuda")
    order = rng.permutation(n)
    table = np.full((len(tokens), max(need + [1])), -1, np.int32)
    a = 0
    for b, k in enumerate(need):
        table[b, :k] = order[a:a + k]
        a += k
    return hf.PagedKV(pages, torch.as_tensor(table, device="cuda"), H, d, P), table


def _unpacked(cache, layer=0):
    pages = cache.pages[layer].cpu().numpy()
    return {p: at.unpack_page(pages[p], cache.H, cache.d_h, cache.page_tokens)
            for p in range(pages.shape[0])}


@pytest.mark.parametrize("d,P", [(64, 32), (128, 32), (128, 64), (64, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("start,n", [([0], [1]), ([0], [64]), ([31, 0, 5], [1, 70, 3]),
                                     ([33, 64, 7], [40, 0, 26])],
                         ids=["one", "two blocks", "ragged", "inside"])
def test_append_codes_bit_for_bit(torch, d, P, dtype, start, n):
    from paper_2609_32259_amd import heterofold as hf
    L, H = 2, 3
    print(f"[gpu-paged] append {dtype} d={d} P={P} start={start} n={n}", flush=True)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    cache, table = _cache(torch, [a + b for a, b in zip(start, n)], L, H, d, P, 1)
    before = [_unpacked(cache, l) for l in range(L)]
    g = torch.Generator().manual_seed(2)
    kv = torch.randn((len(n), L, 2, H, max(max(n), 1) + 2, d), generator=g)
    kv = (kv * torch.exp(torch.randn(d, generator=g))).to(t)
    kv[..., :32] = kv[..., :1]            # a group without spread
    kv[0, 0, 0, 1, 0, 40] = math.nan      # and ones that are not finite
    kv[0, 0, 1, 2, 0, 33] = -math.inf
    dev = kv.cuda()
    hf.hf_paged_append(cache, start, n, dev[:, :, 0], dev[:, :, 1])
    torch.cuda.synchronize()
    x = kv.float().numpy()
    for l in range(L):
        after = _unpacked(cache, l)
        want = {p: tuple(y.copy() for y in u) for p, u in before[l].items()}
        for b in range(len(n)):
            for i in range(n[b]):
                tok = start[b] + i
                p, r = int(table[b, tok // P]), tok % P
                for role in range(2):
                    c, s, o = at.quantise(x[b, l, role, :, i])
                    want[p][0][role, r], want[p][1][role, r], want[p][2][role, r] = c, s, o
        for p in want:
            for y, z, name in zip(after[p], want[p], ("codes", "scales", "offsets")):
                assert np.array_equal(np.asarray(y).view(np.uint8 if name == "codes" else np.uint32)
                                      if name == "codes" else np.nan_to_num(y, nan=9e9),
                                      np.asarray(z).view(np.uint8) if name == "codes"
                                      else np.nan_to_num(z, nan=9e9)), (l, p, name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,theta,pos0", [([1, 1], 1.0e4, [0, 30000]), ([45, 4], 5.0e5, [0, 7]),
                                          ([130, 6], 1.0e9, [100000, 0])],
                         ids=["step", "short", "long"])
def test_append_rotates_keys(torch, dtype, d, n, theta, pos0):
    from paper_2609_32259_amd import heterofold as hf
    H, P, start = 2, 64, [37, 3]
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    cache, table = _cache(torch, [a + b for a, b in zip(start, n)], 1, H, d, P, 3)
    g = torch.Generator().manual_seed(4)
    k = torch.randn((sum(n), H, d), generator=g).to(t)
    v = torch.randn((sum(n), H, d), generator=g).to(t)
    hf.hf_paged_append(cache, start, n, k.cuda(), v.cuda(), theta=theta, pos0=pos0)
    back = [torch.full((sum(n), H, d), 9.0, device="cuda") for _ in range(2)]
    hf.hf_paged_read(cache, start, n, *back)
    torch.cuda.synchronize()
    a = 0
    for b in range(2):
        pos = pos0[b] + start[b] + np.arange(n[b])
        x = f64(k[a:a + n[b]]).transpose(1, 0, 2)
        x = ro.rotate(x, pos, theta).transpose(1, 0, 2)
        for want, got, noise in ((x, back[0], 1), (f64(v[a:a + n[b]]), back[1], 0)):
            y = want.reshape(n[b], H, -1, 32)
            lo, hi = y.min(-1, keepdims=True), y.max(-1, keepdims=True)
            # half a step of 15 (of the rounded spread), what the rounding of o and s leaves at the
            # ends, and the fp32 rotation: cos, sin, two products and a sum of a pair
            amp = np.abs(y).max(-1, keepdims=True)
            lim = (hi - lo) / 30 * (1 + UB) + UB * (np.abs(lo) + (hi - lo)) + noise * 8 * U32 * amp * 2 + 4 * U32 * amp
            err = np.abs(f64(got[a:a + n[b]]).reshape(y.shape) - y)
            assert (err <= lim).all(), float((err / lim).max())
        a += n[b]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,P", [(64, 64), (128, 128)])
def test_read_gives_the_values(torch, dtype, d, P):
    from paper_2609_32259_amd import heterofold as hf
    L, H, start, n = 3, 2, [0, 45, 130], [150, 1, 33]
    cache, table = _cache(torch, [a + b for a, b in zip(start, n)], L, H, d, P, 5)
    table[0, 0] = -1                                        # holes
    table[2, -1] = cache.pages.shape[1]
    cache.table.copy_(torch.as_tensor(table))
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    out = torch.full((3, 2, 2, H, 160, d), 7.0, dtype=t, device="cuda")
    hf.hf_paged_read(cache, start, n, out[:, :, 0], out[:, :, 1], layer=1)
    torch.cuda.synchronize()
    got = f64(out)
    for l in (1, 2):
        codes = _unpacked(cache, l)
        for b in range(3):
            c, s, o, seen = logical(table, codes, H, d, P, b, start[b] + n[b])
            with np.errstate(invalid="ignore", over="ignore"):
                x = at.dequantise(c, s, o)[:, start[b]:]
                x[:, ~seen[start[b]:]] = 0
                x = x.astype(np.float32)
                if dtype == "bf16":
                    x = at._bf16(x)
            w = got[b, l - 1, :, :, :n[b]].transpose(0, 2, 1, 3)
            assert np.array_equal(np.nan_to_num(x, nan=1.5, posinf=3e38, neginf=-3e38),
                                  np.nan_to_num(w.astype(np.float32), nan=1.5, posinf=3e38, neginf=-3e38))
            assert (got[b, l - 1, :, :, n[b]:] == 7).all()


def _fill(torch, cache, table, tokens, seed, sigma=0.5):
    """Ordinary rows in every token of the table, garbage behind."""
    from paper_2609_32259_amd import heterofold as hf
    g = torch.Generator().manual_seed(seed)
    H, d = cache.H, cache.d_h
    x = torch.randn((2, sum(tokens), H, d), generator=g) * torch.exp(sigma * torch.randn(d, generator=g))
    for l in range(cache.L):
        hf.hf_paged_append(cache, [0] * len(tokens), tokens, x[0].cuda(), x[1].cuda(), layer=l)


def _attend(torch, dtype, q_len, kv_len, Hq, H, d, P, causal=True, seed=0, holes=(), layer=0, L=1,
            **kw):
    from paper_2609_32259_amd import heterofold as hf
    print(f"[gpu-paged] attend {dtype} q={q_len} kv={kv_len} heads {Hq}/{H} d={d} P={P} "
          f"holes={holes}", flush=True)
    cache, table = _cache(torch, kv_len, L, H, d, P, seed)
    _fill(torch, cache, table, kv_len, seed)
    for b, j, p in holes:
        table[b, j] = p
    cache.table.copy_(torch.as_tensor(table))
    g = torch.Generator().manual_seed(seed + 9)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = (1.5 * torch.randn((sum(q_len), Hq, d), generator=g)).to(t).cuda()
    out, lse = hf.hf_paged_attention(q, cache, q_len, kv_len, layer=layer, causal=causal,
                                     return_lse=True, **kw)
    torch.cuda.synchronize()
    codes = _unpacked(cache, layer)
    a = 0
    for b, n in enumerate(q_len):
        c, s, o, seen = logical(table, codes, H, d, P, b, kv_len[b])
        c, s, o = (np.where(seen[:, None, None], x, 0) for x in (c, s, o))
        x = at.dequantise(c, s, o)
        qq = f64(q[a:a + n])
        ref = at.attend(qq, x[0], x[1], 1 / math.sqrt(d), causal, seen)
        # magnitudes of what is summed: codes enter the products as 16 + code <= 31, taken out
        # again by numbers of up to |o| + 16 s, and as code - 8 beside |o| + 8 s
        rep = lambda y: np.repeat(y.astype(np.float64), 32, axis=-1)  # noqa: E731
        big_k = rep(47 * s[0] + np.abs(o[0]))
        arg = np.array([[(np.abs(qq[i, h]) @ big_k[ref["weights"][i, h][0], h // (Hq // H)].T).max()
                         / math.sqrt(d) if (i, h) in ref["weights"] else 0.0
                         for h in range(Hq)] for i in range(n)]).reshape(n, Hq)
        mean = lambda y: np.array([[ref["weights"][i, h][1] @ y[ref["weights"][i, h][0], h // (Hq // H)]  # noqa: E731
                                    if (i, h) in ref["weights"] else np.zeros(d)
                                    for h in range(Hq)] for i in range(n)]).reshape(n, Hq, d)
        big_v = mean(rep(64 * s[1] + np.abs(o[1])))
        bo, bl = bounds(ref, d, kv_len[b], "f32", mag=big_v, arg=arg)
        # (bounds() of "f32": the three bf16 terms of a weight hold 24 bits, one half step more)
        bo = bo + U32 * big_v
        if dtype == "bf16":   # the weight times the scale, against code - 8; the result
            bo = bo + UB * mean(rep(8 * s[1]))
            bo = bo + UB * (np.abs(ref["out"]) + bo)
        check(f64(out[a:a + n]), ref["out"], bo, f"out of sequence {b}")
        check(f64(lse[a:a + n]), ref["lse"], bl, f"lse of sequence {b}")
        a += n


CASES = [
    # q_len, kv_len, Hq, H, P
    ([1], [1], 1, 1, 32),
    ([1], [33], 8, 1, 64),
    ([1, 1, 1], [64, 127, 300], 10, 2, 64),
    ([4], [4], 4, 2, 32),
    ([5, 1], [90, 31], 7, 1, 32),
    ([3, 0, 2], [130, 9, 2], 4, 4, 128),
    ([16], [200], 8, 2, 256),
    ([21], [75], 5, 1, 64),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_against_the_oracle(torch, dtype, d, case):
    q_len, kv_len, Hq, H, P = CASES[case]
    _attend(torch, dtype, q_len, kv_len, Hq, H, d, P, seed=case, L=2, layer=case % 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_masks(torch, dtype):
    _attend(torch, dtype, [9, 20], [130, 33], 6, 2, 64, 32, causal=False)
    _attend(torch, dtype, [9, 3, 70, 4], [2, 0, 65, 4], 4, 2, 128, 64)      # rows that see nothing
    _attend(torch, dtype, [1, 3], [150, 70], 4, 2, 128, 32,
            holes=[(0, 0, -1), (0, 3, 1 << 30), (1, 2, -5)])
    _attend(torch, dtype, [2, 2], [64, 64], 4, 2, 64, 32,
            holes=[(0, 0, -1), (0, 1, -1), (1, 1, 99999)])                   # nothing, and half


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("q_len,kv_len,Hq,H", [([1], [4001], 4, 1), ([2, 1], [2100, 500], 6, 2)],
                         ids=["token", "tokens"])
def test_attention_split(torch, dtype, d, q_len, kv_len, Hq, H):
    from paper_2609_32259_amd import heterofold as hf
    code = hf.HF_BF16 if dtype == "bf16" else hf.HF_F32
    assert hf.hf_attention_workspace_bytes(q_len, kv_len, Hq, H, d, code, paged=True) > 0
    _attend(torch, dtype, q_len, kv_len, Hq, H, d, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_not_seen_has_no_influence(torch, dtype):
    """Groups that are not finite reach the rows that see them and no other."""
    from paper_2609_32259_amd import heterofold as hf
    H, d, P, n, t, Hq = 2, 128, 32, 4, 70, 4
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    cache, table = _cache(torch, [t], 1, H, d, P, 6)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((t, H, d), generator=g).cuda() for _ in range(2))
    q = torch.randn((n, Hq, d), generator=g).to(td).cuda()
    hf.hf_paged_append(cache, [0], [t], k, v)
    ref, lse = hf.hf_paged_attention(q, cache, [n], [t], return_lse=True)
    for what in (0, 1):
        for row in (1, n - 1):
            x = [k[t - n + row:t - n + row + 1].clone(), v[t - n + row:t - n + row + 1].clone()]
            x[what][0, 1, 40] = math.nan
            hf.hf_paged_append(cache, [t - n + row], [1], *x)
            out, l2 = hf.hf_paged_attention(q, cache, [n], [t], return_lse=True)
            torch.cuda.synchronize()
            assert torch.equal(out[:, :2], ref[:, :2]) and torch.equal(out[:row], ref[:row])
            assert torch.equal(l2[:row], lse[:row])
            if what == 0:
                assert bool(torch.isnan(out[row:, 2:].float()).all())
            else:
                assert bool(torch.isnan(out[row:, 2:, 32:64].float()).all())
                keep = [e for e in range(d) if not 32 <= e < 64]
                assert torch.equal(out[:, :, keep], ref[:, :, keep])
            hf.hf_paged_append(cache, [t - n + row], [1], k[t - n + row:t - n + row + 1],
                               v[t - n + row:t - n + row + 1])
    assert torch.equal(hf.hf_paged_attention(q, cache, [n], [t]), ref)


def test_holes_drop_rows_and_shared_pages_are_read(torch):
    from paper_2609_32259_amd import heterofold as hf
    H, d, P = 2, 64, 32
    cache, table = _cache(torch, [96, 96], 1, H, d, P, 7)
    _fill(torch, cache, table, [96, 96], 8)
    table[1, :2] = table[0, :2]            # a shared prefix
    table[0, 2] = -1
    cache.table.copy_(torch.as_tensor(table))
    before = cache.pages.clone()
    x = torch.randn((20, H, d), device="cuda")
    hf.hf_paged_append(cache, [70, 0], [20, 0], x, x)
    assert torch.equal(cache.pages, before)
    q = torch.randn((1, 4, d), device="cuda").bfloat16().repeat(2, 1, 1)
    out = hf.hf_paged_attention(q, cache, [1, 1], [64, 64])
    assert torch.equal(out[0], out[1])


def test_a_receivers_turn_together(torch):
    """A cache goes into pages, a question is answered over them, tokens are appended and
    decoded one by one, and the rows come back dense for the next hand-off: attention over
    the pages agrees with attention over the rows read back, step by step, eager and in a
    graph."""
    from paper_2609_32259_amd import heterofold as hf
    H, Hq, d, P, L, T, n = 8, 40, 128, 64, 2, 301, 9
    theta = 5.0e5
    g = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    cache, table = _cache(torch, [T + n], L, H, d, P, 12)
    R = rnd(1, L, 2, H, T, d)
    hf.hf_paged_append(cache, [0], [T], R[:, :, 0], R[:, :, 1])
    dense = torch.zeros((1, L, 2, H, T + n, d), device="cuda")
    at_ = T
    for m in (4, 1, 1, 1, 1, 1):                      # the question, then tokens
        k, v, q = rnd(m, H, d), rnd(m, H, d), rnd(m, Hq, d)
        for l in range(L):
            hf.hf_paged_append(cache, [at_], [m], k, v, theta=theta, layer=l)
        at_ += m
        hf.hf_paged_read(cache, [0], [at_], dense[:, :, 0], dense[:, :, 1])
        for l in range(L):
            got, lse = hf.hf_paged_attention(q, cache, [m], [at_], layer=l, return_lse=True)
            want, lse2 = hf.hf_prompt_attention(q.float(), dense[:, l, 0], dense[:, l, 1], [m], [at_],
                                                return_lse=True)
            # bf16 weights of about sqrt(sum w^2) x the values, and the result's rounding: within
            # two half steps of the largest value
            lim = 2 * UB * float(dense[:, l, 1].abs().max())
            assert float((got.float() - want).abs().max()) <= lim
            assert float((lse - lse2).abs().max()) <= 1e-4
    # one decoding step captured: append and attention replay on new rows
    k, v, q = rnd(1, H, d), rnd(1, H, d), rnd(1, Hq, d)

    def step():
        hf.hf_paged_append(cache, [at_ - 1], [1], k, v, theta=theta, layer=1)
        return hf.hf_paged_attention(q, cache, [1], [at_], layer=1)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        for x in (k, v, q):
            x.copy_(rnd(*x.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step()), i


def test_two_streams(torch):
    from paper_2609_32259_amd import heterofold as hf
    runs = []
    for s in range(2):
        cache, table = _cache(torch, [900, 333], 1, 2, 128, 64, 20 + s)
        _fill(torch, cache, table, [900, 333], 30 + s)
        q = torch.randn((2, 8, 128), device="cuda").bfloat16()
        runs.append((q, cache, hf.hf_paged_attention(q, cache, [1, 1], [900, 333])))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [hf.hf_paged_attention(q, c, [1, 1], [900, 333], stream=s)
               for _ in range(2) for (q, c, _), s in zip(runs, streams)]
        torch.cuda.synchronize()
        for i, o in enumerate(got):
            assert torch.equal(o, runs[i % 2][2])
