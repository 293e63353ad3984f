"""Packed and paged attention, writing and reading a paged cache, where single steps of them go wrong.  Tolerances as in test_gpu_serving.py unless a test
derives its own."""
import numpy as np
import pytest
import torch

from test_gpu_serving import atp, host, ints  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ rounding of wide scores in fp32
def _sums(q, k, group, mid):
    """Scores in fp32: chains of fused products over `group` features, added up over `mid` features, those added up.  A chain takes a feature of the first and
    one of the second four of eight in turn."""
    f = np.float32
    total = np.zeros(len(q), f)
    for t in range(0, 256, mid):
        part = np.zeros(len(q), f)
        for u in range(t, t + mid, group):
            s = np.zeros(len(q), f)
            for w in range(u, u + group, 8):
                for c in (w, w + 4, w + 1, w + 5, w + 2, w + 6, w + 3, w + 7):
                    s = (q[:, c].astype(np.float64) * k[:, c] + s).astype(f)
            part = part + s
        total = total + part
    return total.astype(np.float64)


def test_scores_of_256_features_in_fp32_are_short_sums(atp):
    """Two keys a sequence that differ by little, with values 1 and 0: O = 1 / (1 + exp(s1 - s0)), scale 1, and the scores are so large (standard deviation
    256) that their rounding is all that counts: the error of O over O·(1 - O) is that of s1 - s0.  Sums of 8 features, added up over 64, leave 0.80 of
    what sums of 16 in one row leave; the bound is 1.07 times the former, on these very inputs (2^12 rows: the mean square is good to 2.2 %, its root to 1.1 %)."""
    rng = np.random.default_rng(71)
    n, d = 1 << 12, 256
    q = rng.standard_normal((n, d)).astype(np.float32)
    k0 = (16 * rng.standard_normal((n, d))).astype(np.float32)
    k1 = k0 + (rng.standard_normal((n, d)) / 32).astype(np.float32)
    exact = (q.astype(np.float64) * (k1.astype(np.float64) - k0)).sum(-1)
    mean = lambda x: np.sqrt((x ** 2).mean())  # noqa: E731
    short, long = (mean(_sums(q, k1, *o) - _sums(q, k0, *o) - exact) for o in ((8, 64), (16, 256)))
    assert long > 1.15 * short
    Q, K, V = (np.zeros((2 * n, 1, d), np.float32) for _ in range(3))
    Q[::2, 0], Q[1::2, 0], K[::2, 0], K[1::2, 0], V[::2] = q, q, k0, k1, 1.0
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    want = 1 / (1 + np.exp(exact))
    table = np.arange(2 * n).reshape(n, 2)[:, ::-1].copy()
    cache = atp.PagedCache.empty(2 * n, 1, 1, d, torch.float32)
    args = (ints(table), ints([2] * n), ints(2 * np.arange(n + 1)))
    atp.cache_write(cache, dev(K), dev(V), *args)
    for got in (atp.attention_packed(dev(Q), dev(K), dev(V), args[2], causal=False, scale=1.0), atp.attention_paged(dev(Q), cache, *args, causal=False, scale=1.0)):
        off = (host(got)[::2, 0, 0] - want) / (want * (1 - want))
        print(f"scores off by {mean(off):.3e}, short sums {short:.3e}, long {long:.3e}", flush=True)
        assert mean(off) <= 1.07 * short
