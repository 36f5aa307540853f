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
