"""GPU: hf_prompt_attention against the fp64 oracle, element by element within the
bounds of ``_attention``: head layouts, lengths from one token up, odd sizes, packed
rows and cache views, rows that see nothing, what lies in masked places, split key
ranges, and calls on other streams and in graphs."""

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


def _inputs(torch, dtype, q_len, kv_len, Hq, H, d, seed, layout):
    g = torch.Generator().manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = (1.5 * torch.randn((sum(q_len), Hq, d), generator=g)).to(t)
    if layout == "cache":
        kv = torch.randn((len(kv_len), 3, 2, H, max(kv_len) + 5, d), generator=g).to(t)
        for b, n in enumerate(kv_len):
            kv[b, :, :, :, n:] = math.nan    # behind the sequence
        kv = kv.cuda()
        k, v = kv[:, 1, 0], kv[:, 1, 1]
        seqs = [(k[b, :, :n].transpose(0, 1), v[b, :, :n].transpose(0, 1))
                for b, n in enumerate(kv_len)]
    else:   # a fused projection: keys and values beside each other in one row
        kv = torch.randn((sum(kv_len) + 3, 2 * H + 1, d), generator=g).to(t)
        kv[sum(kv_len):] = math.nan
        kv = kv.cuda()
        k, v = kv[:, :H], kv[:, H:2 * H]
        at_, seqs = 0, []
        for n in kv_len:
            seqs.append((k[at_:at_ + n], v[at_:at_ + n]))
            at_ += n
    return q.cuda(), k, v, seqs


def _run(torch, dtype, q_len, kv_len, Hq, H, d, causal=True, seed=0, layout="packed", scale=None,
         **kw):
    from paper_2609_32259_amd import heterofold as hf
    print(f"[gpu-attention] {dtype} q={q_len} kv={kv_len} heads {Hq}/{H} d={d} causal={causal} "
          f"{layout}", flush=True)
    q, k, v, seqs = _inputs(torch, dtype, q_len, kv_len, Hq, H, d, seed, layout)
    out, lse = hf.hf_prompt_attention(q, k, v, q_len, kv_len, causal=causal, scale=scale,
                                      return_lse=True, **kw)
    torch.cuda.synchronize()
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    a = 0
    for b, n in enumerate(q_len):
        ref = at.attend(f64(q[a:a + n]), f64(seqs[b][0]), f64(seqs[b][1]), scale, causal)
        bo, bl = bounds(ref, d, kv_len[b], dtype)
        check(f64(out[a:a + n]), ref["out"], bo, f"out of sequence {b}")
        check(f64(lse[a:a + n]), ref["lse"], bl, f"lse of sequence {b}")
        a += n


CASES = [
    # q_len, kv_len, Hq, H
    ([1], [1], 1, 1),
    ([1], [77], 8, 1),
    ([5], [5], 3, 3),
    ([33], [33], 4, 2),
    ([1, 1, 1], [1, 64, 65], 10, 2),
    ([64], [64], 5, 1),
    ([65, 1, 130], [65, 1, 130], 7, 1),
    ([7, 3], [200, 31], 8, 2),
    ([40], [171], 14, 2),
    ([3, 0, 2], [130, 9, 2], 4, 4),
    ([257], [300], 2, 2),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_oracle(torch, dtype, d, case):
    q_len, kv_len, Hq, H = CASES[case]
    layout = "cache" if case % 2 else "packed"
    _run(torch, dtype, q_len, kv_len, Hq, H, d, seed=case, layout=layout)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_not_causal(torch, dtype):
    _run(torch, dtype, [9, 40], [130, 33], 6, 2, 64, causal=False, layout="cache")
    _run(torch, dtype, [70], [50], 6, 2, 128, causal=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["packed", "cache"])
def test_rows_that_see_no_key(torch, dtype, layout):
    _run(torch, dtype, [9, 3, 70, 4], [2, 0, 65, 4], 4, 2, 128, layout=layout)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(torch, dtype):
    """Scores in the hundreds: the running maximum is raised again and again."""
    _run(torch, dtype, [50], [333], 4, 1, 128, scale=3.0)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 64)])
@pytest.mark.parametrize("q_len,kv_len,Hq,H", [([1], [5001], 4, 1), ([2, 1], [3000, 900], 6, 2),
                                               ([40], [4099], 8, 1)],
                         ids=["token", "tokens", "suffix"])
def test_split_key_ranges(torch, dtype, d, q_len, kv_len, Hq, H):
    from paper_2609_32259_amd import heterofold as hf
    code = hf.HF_BF16 if dtype == "bf16" else hf.HF_F32
    assert hf.hf_attention_workspace_bytes(q_len, kv_len, Hq, H, d, code) > 0
    _run(torch, dtype, q_len, kv_len, Hq, H, d, layout="cache")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 100], ids=["short", "long"])
def test_what_is_not_seen_has_no_influence(torch, dtype, n):
    """Keys and values that are not finite reach the rows that see them and no other."""
    from paper_2609_32259_amd import heterofold as hf
    d, Hq, H, t = 128, 4, 2, 150
    q, k, v, _ = _inputs(torch, dtype, [n], [t], Hq, H, d, 3, "packed")
    k, v = k[:t].clone(), v[:t].clone()
    ref, lse = hf.hf_prompt_attention(q, k, v, [n], [t], return_lse=True)
    first = t - n                       # row i sees keys up to first + i
    for what, bad in (("v", math.nan), ("v", math.inf), ("k", math.nan), ("k", math.inf)):
        for row in (1, n - 1):
            k2, v2 = k.clone(), v.clone()
            (v2 if what == "v" else k2)[first + row, 1, 5] = bad
            out, l2 = hf.hf_prompt_attention(q, k2, v2, [n], [t], return_lse=True)
            torch.cuda.synchronize()
            assert torch.equal(out[:, :2], ref[:, :2])            # the other key/value head
            assert torch.equal(out[:row, 2:], ref[:row, 2:]), (what, bad, row)
            assert torch.equal(l2[:row], lse[:row])
            if what == "v":
                got = out[row:, 2:, 5].float()
                assert bool(torch.isnan(got).all() if bad != bad else (got == math.inf).all())
                keep = [e for e in range(d) if e != 5]
                assert torch.equal(out[:, :, keep], ref[:, :, keep])
            elif bad != bad:
                assert bool(torch.isnan(out[row:, 2:].float()).all())


def test_rows_outside_the_call_keep_their_bits(torch):
    from paper_2609_32259_amd import heterofold as hf
    for dtype, q_len, kv_len in (("bf16", [5, 2], [40, 3]), ("f32", [1, 3], [700, 3]),
                                 ("bf16", [1], [5000])):
        q, k, v, _ = _inputs(torch, dtype, q_len, kv_len, 4, 2, 64, 1, "packed")
        n = sum(q_len)
        q = torch.cat([q, q[:1], q[:1]])
        big = torch.full((n + 2, 4, 80), 7.0, dtype=q.dtype, device="cuda")
        out = big[:, :, :64]
        lse = torch.full((n + 2, 4), 7.0, device="cuda")
        ref = hf.hf_prompt_attention(q[:n].contiguous(), k, v, q_len, kv_len)
        hf.hf_prompt_attention(q, k, v, q_len, kv_len, out=out, lse=lse)
        torch.cuda.synchronize()
        assert torch.equal(out[:n], ref)
        assert bool((big[n:] == 7).all()) and bool((big[:, :, 64:] == 7).all())
        assert bool((lse[n:] == 7).all()) and bool((lse[:n] != 7).all())


def test_in_place(torch):
    from paper_2609_32259_amd import heterofold as hf
    for q_len, kv_len in (([70, 9], [70, 200]), ([1], [4000])):
        q, k, v, _ = _inputs(torch, "bf16", q_len, kv_len, 8, 2, 128, 5, "packed")
        ref = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
        got = hf.hf_prompt_attention(q, k, v, q_len, kv_len, out=q)
        assert got is q and torch.equal(got, ref)


@pytest.mark.parametrize("q_len,kv_len", [([90], [90]), ([1, 1], [3000, 77])],
                         ids=["prompt", "tokens"])
def test_streams_and_graphs(torch, q_len, kv_len):
    """Two calls with workspaces of their own on two streams, and a captured call that
    replays on new contents of its inputs."""
    from paper_2609_32259_amd import heterofold as hf
    ins = [_inputs(torch, "bf16", q_len, kv_len, 8, 2, 128, s, "cache")[:3] for s in (1, 2)]
    ref = [hf.hf_prompt_attention(*x, q_len, kv_len) for x in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rnd in range(3):
        got = [hf.hf_prompt_attention(*x, q_len, kv_len, stream=s)
               for _ in range(2) for x, s in zip(ins, streams)]
        torch.cuda.synchronize()
        for i, o in enumerate(got):
            assert torch.equal(o, ref[i % 2]), (rnd, i)
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
        assert torch.equal(out, ref[i])


def test_same_result_every_time(torch):
    from paper_2609_32259_amd import heterofold as hf
    for q_len, kv_len in (([300], [300]), ([1], [9000]), ([100], [6000])):
        q, k, v, _ = _inputs(torch, "bf16", q_len, kv_len, 8, 2, 128, 9, "packed")
        ref = hf.hf_prompt_attention(q, k, v, q_len, kv_len)
        for _ in range(3):
            assert torch.equal(hf.hf_prompt_attention(q, k, v, q_len, kv_len), ref)


def test_keys_past_four_gigabytes(torch):
    """Rows 64 KiB apart: the last keys lie past 32-bit byte offsets."""
    from paper_2609_32259_amd import heterofold as hf
    t, stride = 70_000, 32768
    buf = torch.empty(t * stride, dtype=torch.bfloat16, device="cuda")
    rows = buf.view(t, stride)
    g = torch.Generator(device="cuda").manual_seed(0)
    kv = torch.randn((t, 2, 128), generator=g, device="cuda").bfloat16()
    rows[:, :256] = kv.view(t, 256)
    k, v = rows[:, None, :128], rows[:, None, 128:256]
    q = torch.randn((3, 4, 128), generator=g, device="cuda").bfloat16()
    got = hf.hf_prompt_attention(q, k, v, [3], [t])
    ref = hf.hf_prompt_attention(q, kv[:, :1].contiguous(), kv[:, 1:].contiguous(), [3], [t])
    assert torch.equal(got, ref)
    q = torch.randn((80, 2, 128), generator=g, device="cuda").bfloat16()
    got = hf.hf_prompt_attention(q, k, v, [80], [t])
    ref = hf.hf_prompt_attention(q, kv[:, :1].contiguous(), kv[:, 1:].contiguous(), [80], [t])
    assert torch.equal(got, ref)
