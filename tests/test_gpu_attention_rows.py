"""GPU: prompt attention by rows -- tiles of 256 query rows that fill the chip, which the
planner takes for any lengths where they are at least as many as its workgroups (256): that
is checked here from the lengths, so no change of its estimates moves a case to the other
kernel.  Values, keys and queries that are not finite in either stage of the keys, and the
call's forms (in place, strided results, streams, graphs, far rows) on that kernel."""

import math

import numpy as np
import pytest

from _attention import bounds, check
from oracle import attention as at

pytestmark = pytest.mark.gpu

ROWS = {"bf16": 256, "f32": 64}      # query rows of a workgroup's tile
FILL = 256                           # workgroups that fill the chip


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU test needs a GPU"
    from paper_2609_32259_amd import heterofold
    heterofold.lib()
    return torch


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _by_rows(dtype, q_len, kv_len, Hq, H, d, split=False):
    """The lengths are those of a call by rows; split: with cut key ranges, or not."""
    from paper_2609_32259_amd import heterofold as hf
    tiles = sum(-(-n * (Hq // H) // ROWS[dtype]) for n in q_len) * H
    assert tiles >= FILL and max(q_len) * (Hq // H) > 32, (tiles, q_len)
    code = hf.HF_BF16 if dtype == "bf16" else hf.HF_F32
    assert (hf.hf_attention_workspace_bytes(q_len, kv_len, Hq, H, d, code) > 0) == split


def _draw(torch, dtype, q_len, kv_len, Hq, H, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rnd = lambda n, h: torch.randn((n, h, d), generator=g, device="cuda").to(t)  # noqa: E731
    return 1.5 * rnd(sum(q_len), Hq), rnd(sum(kv_len), H), rnd(sum(kv_len), H)


def _lengths(seed, B, lo, hi, cache=0):
    rng = np.random.default_rng(seed)
    q_len = [int(x) for x in rng.integers(lo, hi + 1, size=B)]
    return q_len, [n + int(rng.integers(0, cache + 1)) for n in q_len]


def _bits(torch, x):
    return x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)


# Sequences of several tiles of rows each: (G, H, d, lengths' range, keys before the prompt).
BATCHES = [
    (1, 6, 128, 24, (320, 600), 0),
    (1, 8, 64, 24, (257, 300), 90),
    (4, 3, 128, 10, (512, 600), 0),
    (4, 4, 64, 16, (256, 330), 200),
]


@pytest.mark.parametrize("G,H,d,B,span,cache", BATCHES, ids=["G1-128", "G1-64", "G4-128", "G4-64"])
def test_bad_values_and_keys_in_every_tile(torch, G, H, d, B, span, cache):
    """One value or key that is not finite, in turn in every tile of 64 keys (so that the tiles
    after it end in either stage): all rows that do not see it keep their bits, those that see a
    value get it, and those that see a key that is NaN are NaN."""
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len = _lengths(1, B, *span, cache=cache)
    _by_rows("bf16", q_len, kv_len, G * H, H, d)
    q, k, v = _draw(torch, "bf16", q_len, kv_len, G * H, H, d, 2)
    ref, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    b = B // 2
    n, t = q_len[b], kv_len[b]
    q0, k0 = sum(q_len[:b]), sum(kv_len[:b])
    print(f"[gpu-attention-rows] tiles G={G} H={H} d={d} n={n} t={t}", flush=True)
    bads = [("v", math.nan), ("v", math.inf), ("v", -math.inf), ("k", math.nan)]
    for tile in range(-(-t // 64)):
        last = min(64 * tile + 63, t - 1)
        for i, key in enumerate((64 * tile, (64 * tile + last) // 2, last)):
            what, bad = bads[(tile + i) % 4]
            x = v if what == "v" else k
            was = x[k0 + key, 1, 37].clone()
            x[k0 + key, 1, 37] = bad
            out, l2 = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
            x[k0 + key, 1, 37] = was
            torch.cuda.synchronize()
            row = max(0, key - (t - n))      # the first that sees it
            hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
            hit[q0 + row:q0 + n, G:2 * G, 37 if what == "v" else slice(None)] = True
            same = _bits(torch, out) == _bits(torch, ref)
            assert bool((same | hit).all()), (what, bad, key, int((~(same | hit)).sum()))
            got = out[hit].float()
            assert bool((torch.isnan(got) if bad != bad else got == bad).all()), (what, bad, key)
            keep = torch.ones(l2.shape, dtype=torch.bool, device="cuda")
            if what == "k":
                keep[q0 + row:q0 + n, G:2 * G] = False
            assert torch.equal(l2[keep], lse[keep]), (what, bad, key)


@pytest.mark.parametrize("G,H,d,B,span,cache", BATCHES, ids=["G1-128", "G1-64", "G4-128", "G4-64"])
def test_bad_queries_in_every_wave(torch, G, H, d, B, span, cache):
    """A query that is not finite makes its workgroup compute a second time: every other row keeps
    its bits."""
    from paper_2609_32259_amd import heterofold as hf
    q_len, kv_len = _lengths(3, B, *span, cache=cache)
    _by_rows("bf16", q_len, kv_len, G * H, H, d)
    q, k, v = _draw(torch, "bf16", q_len, kv_len, G * H, H, d, 4)
    ref = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
    torch.cuda.synchronize()
    b = B // 3
    n, q0 = q_len[b], sum(q_len[:b])
    for token in range(0, n, 29):
        head = token % (G * H)
        was = q[q0 + token, head, 5].clone()
        q[q0 + token, head, 5] = math.nan if token % 2 else math.inf
        out = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
        q[q0 + token, head, 5] = was
        torch.cuda.synchronize()
        hit = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
        hit[q0 + token, head] = True
        assert bool(torch.isnan(out[hit].float()).all()), token
        assert torch.equal(_bits(torch, out)[~hit], _bits(torch, ref)[~hit]), token


# 24 sequences of one to three tiles of 256 rows, odd lengths and a cache before some
FORM = dict(Hq=24, H=8, span=(65, 190), B=24, cache=70)


def _form(torch, dtype, d, seed):
    q_len, kv_len = _lengths(5, FORM["B"], *FORM["span"], cache=FORM["cache"])
    _by_rows(dtype, q_len, kv_len, FORM["Hq"], FORM["H"], d)
    return (*_draw(torch, dtype, q_len, kv_len, FORM["Hq"], FORM["H"], d, seed), q_len, kv_len)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_against_the_oracle_and_in_place(torch, dtype, d):
    from paper_2609_32259_amd import heterofold as hf
    q, k, v, q_len, kv_len = _form(torch, dtype, d, 6)
    print(f"[gpu-attention-rows] in place {dtype} d={d}", flush=True)
    out, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    torch.cuda.synchronize()
    a = c = 0
    for b, (n, t) in enumerate(zip(q_len, kv_len)):
        if b in (0, 11, 23):
            ref = at.attend(f64(q[a:a + n, 3:6]), f64(k[c:c + t, 1:2]), f64(v[c:c + t, 1:2]),
                            1 / math.sqrt(d), True)
            bo, bl = bounds(ref, d, t, dtype)
            check(f64(out[a:a + n, 3:6]), ref["out"], bo, f"out of sequence {b}")
            check(f64(lse[a:a + n, 3:6]), ref["lse"], bl, f"lse of sequence {b}")
        a, c = a + n, c + t
    got = hf.hf_prompt_attention(q, k, v, q_len, kv_len, out=q)
    torch.cuda.synchronize()
    assert got is q and torch.equal(got, out)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_and_channels_outside_the_call_keep_their_bits(torch, dtype, d):
    from paper_2609_32259_amd import heterofold as hf
    q, k, v, q_len, kv_len = _form(torch, dtype, d, 7)
    n, Hq = sum(q_len), FORM["Hq"]
    ref, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, return_lse=True)
    more = torch.cat([q, q[:2]])
    big = torch.full((n + 2, Hq, d + 16), 7.0, dtype=q.dtype, device="cuda")
    l2 = torch.full((n + 2, Hq), 7.0, device="cuda")
    hf.hf_prompt_attention(more, k, v, q_len, kv_len, out=big[:, :, :d], lse=l2)
    torch.cuda.synchronize()
    assert torch.equal(big[:n, :, :d], ref) and torch.equal(l2[:n], lse)
    assert bool((big[n:] == 7).all()) and bool((big[:, :, d:] == 7).all()) and bool((l2[n:] == 7).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch(torch, dtype):
    """Queries, keys and results [B, H, T, d], every sequence shorter than its room; behind
    its length a sequence's queries and keys are NaN and its results stay as they were."""
    from paper_2609_32259_amd import heterofold as hf
    q, k, v, q_len, kv_len = _form(torch, dtype, 128, 8)
    B, Hq, H = FORM["B"], FORM["Hq"], FORM["H"]
    ref = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
    room = max(kv_len) + 3
    pad = lambda h: torch.full((B, h, room, 128), math.nan, dtype=q.dtype, device="cuda")  # noqa: E731
    q4, k4, v4, o4 = pad(Hq), pad(H), pad(H), pad(Hq)
    o4.fill_(7.0)
    a = c = 0
    for b, (n, t) in enumerate(zip(q_len, kv_len)):
        q4[b, :, :n] = q[a:a + n].transpose(0, 1)
        k4[b, :, :t] = k[c:c + t].transpose(0, 1)
        v4[b, :, :t] = v[c:c + t].transpose(0, 1)
        a, c = a + n, c + t
    hf.hf_prompt_attention(q4, k4, v4, q_len, kv_len, out=o4)
    torch.cuda.synchronize()
    a = 0
    for b, n in enumerate(q_len):
        assert torch.equal(o4[b, :, :n], ref[a:a + n].transpose(0, 1)), b
        assert bool((o4[b, :, n:] == 7).all()), b
        a += n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_streams_and_graphs(torch, dtype):
    """Calls on two streams at once, the second with a value that is not finite; then a captured
    call that replays on the contents of either."""
    from paper_2609_32259_amd import heterofold as hf
    ins = [_form(torch, dtype, 128, s)[:3] for s in (9, 10)]
    q_len, kv_len = _form(torch, dtype, 128, 9)[3:]
    ins[1][2][40, 2, 3] = math.inf
    ref = [hf.hf_prompt_attention(*x, q_len, kv_len) for x in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rnd in range(3):
        got = [hf.hf_prompt_attention(*x, q_len, kv_len, stream=s)
               for _ in range(2) for x, s in zip(ins, streams)]
        torch.cuda.synchronize()
        for i, o in enumerate(got):
            assert torch.equal(_bits(torch, o), _bits(torch, ref[i % 2])), (rnd, i)
    q, k, v = (x.clone() for x in ins[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
    for i in (0, 1, 0, 1):
        for dst, src in zip((q, k, v), ins[i]):
            dst.copy_(src)
        out.fill_(5.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(_bits(torch, out), _bits(torch, ref[i])), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_rows_of_keys(torch, dtype):
    """Rows as far apart as the call allows (2^23 elements): the last lie past 32-bit byte
    offsets.  64 sequences read the same keys (a stride of 0 between them)."""
    from paper_2609_32259_amd import heterofold as hf
    t_, n, t, stride = (torch.bfloat16, 256, 300, 1 << 23) if dtype == "bf16" else \
        (torch.float32, 64, 150, 1 << 23)
    B, Hq = 64, 4
    q_len, kv_len = [n] * B, [t] * B
    _by_rows(dtype, q_len, kv_len, Hq, 1, 128)
    g = torch.Generator(device="cuda").manual_seed(11)
    kv = torch.randn((t, 2, 128), generator=g, device="cuda").to(t_)
    q = torch.randn((n * B, Hq, 128), generator=g, device="cuda").to(t_)
    rows = torch.empty((t - 1) * stride + 256, dtype=t_, device="cuda").as_strided((t, 256), (stride, 1))
    rows.copy_(kv.view(t, 256))
    k, v = (rows[None, None, :, 128 * i:128 * (i + 1)].expand(B, -1, -1, -1) for i in range(2))
    got = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
    near = [kv[:, i].contiguous()[None, None].expand(B, -1, -1, -1) for i in range(2)]
    ref = hf.hf_prompt_attention(q, *near, q_len, kv_len)
    torch.cuda.synchronize()
    assert torch.equal(got, ref)
    half = q[:n]
    want = at.attend(f64(half[:, :1]), f64(kv[:, :1]), f64(kv[:, 1:]), 1 / math.sqrt(128), True)
    bo, _ = bounds(want, 128, t, dtype)
    check(f64(got[:n, :1]), want["out"], bo, "out of the first sequence")


def test_same_result_every_time(torch):
    from paper_2609_32259_amd import heterofold as hf
    for dtype in ("bf16", "f32"):
        q, k, v, q_len, kv_len = _form(torch, dtype, 128, 12)
        v[100, 1, 7] = math.nan
        ref = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
        for _ in range(4):
            got = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
            assert torch.equal(_bits(torch, got), _bits(torch, ref))
