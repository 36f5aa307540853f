"""GPU: the bytes of appended pages, all of them: codes, and scales and offsets as the 32-bit
words they are stored in (zeros of either sign, the NaN word, subnormal and largest numbers)."""

import math

import numpy as np
import pytest

from oracle import attention as at

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU test needs a GPU"
    from paper_2609_32259_amd import heterofold
    heterofold.lib()
    return torch


def _groups(rng, dtype):
    """Groups of 32 channels, one a row."""
    r = lambda s=1.0, o=0.0: (rng.standard_normal(32) * s + o)  # noqa: E731
    rows = [r(), r(1e-3, 5.0), r(1e4, -1e6), np.zeros(32), np.full(32, -0.0), np.full(32, 3.25),
            np.full(32, -7.0), r(1e-33), np.abs(r(2e-39)), np.abs(r(1e38)), r(1e30, 1e36),
            np.linspace(-3e38, 3e38, 32),           # spread past the range: NaN
            np.linspace(0.0, 3.2e38, 32), np.linspace(-1.6e38, 1.6e38, 32),
            # quotients halfway between codes: to the even one
            np.concatenate([[0.0, 15.0], np.arange(15) + 0.5, np.arange(15) + 0.5]),
            np.concatenate([[-8.0, 7.0], np.arange(15) - 7.5, np.arange(15) - 7.5])]
    for bad in (math.nan, math.inf, -math.inf):
        x = r()
        x[int(rng.integers(32))] = bad
        rows.append(x)
    if dtype == "f32":
        x = r()
        x[5] = -3.4028e38                            # rounds to -infinity in bf16: NaN
        rows.append(x)
    return np.array(rows, np.float64)


@pytest.mark.parametrize("d,P", [(64, 32), (128, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_byte_for_byte(torch, dtype, d, P):
    from paper_2609_32259_amd import heterofold as hf
    rng = np.random.default_rng(1)
    H, n, start = 3, 77, 21
    g = _groups(rng, dtype)
    pick = rng.integers(0, len(g), size=(2, n, H, d // 32))
    pick.reshape(-1)[:len(g)] = np.arange(len(g))
    x = torch.as_tensor(g[pick].reshape(2, n, H, d).astype(np.float32))
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    n_pages = -(-(start + n) // P) + 1
    before = rng.integers(0, 256, size=(1, n_pages, at.page_bytes(H, d, P)), dtype=np.uint8)
    order = rng.permutation(n_pages)[:n_pages - 1].astype(np.int32)
    cache = hf.PagedKV(torch.as_tensor(before, device="cuda"), torch.as_tensor(order[None], device="cuda"), H, d, P)
    hf.hf_paged_append(cache, [start], [n], x[0].cuda(), x[1].cuda())
    torch.cuda.synchronize()
    got = cache.pages.cpu().numpy()[0]
    y = x.float().numpy()
    want = {int(p): [a.copy() for a in at.unpack_page(before[0, p], H, d, P)] for p in order}
    for i in range(n):
        p, r = int(order[(start + i) // P]), (start + i) % P
        for role in range(2):
            for dst, src in zip(want[p], at.quantise(y[role, i])):
                dst[role, r] = src
    for p in range(n_pages):
        if p not in want:
            assert np.array_equal(got[p], before[0, p]), p
            continue
        bytes_ = at.pack_page(*want[p], H, d, P)
        assert np.array_equal(got[p], bytes_), (p, np.flatnonzero(got[p] != bytes_)[:8])
