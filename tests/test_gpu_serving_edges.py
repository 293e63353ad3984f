"""Packed and paged attention, writing and reading a paged cache, where single steps of them go wrong.  Tolerances as in test_gpu_serving.py unless a test
derives its own."""
import numpy as np
import pytest
import torch

from oracle import serving as so
from test_gpu_serving import TORCH, Pages, atp, check, host, ints, offsets_of, randn  # noqa: F401

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


# ------------------------------------------------------------------ one long sequence among enough rows for the chip
LONG = [
    # dtype, cache, lengths, new tokens, heads, kv_heads, d_h, page size, what max_new says
    ("bf16", "same", [300] * 10 + [9000, 5000], [220] * 10 + [1, 3], 64, 64, 64, 64, 0),                            # row tiles of 128
    ("bf16", "e4m3", [9001] + [250] * 17, [70] + [250] * 17, 32, 16, 128, 16, 0),
    ("bf16", "same", [33] * 400 + [8200], [1] * 401, 64, 64, 64, 32, 1),                                            # of 32
    ("bf16", "e4m3", [20000] + [33] * 400, [2] + [1] * 400, 64, 64, 80, 64, 0),
    ("f32", "same", [9000] + [300] * 5, [5] + [300] * 5, 48, 48, 64, 64, 0),                                        # fp32, of 128
    ("f32", "e4m3", [60] * 80 + [12345], [2] * 80 + [1], 256, 256, 64, 32, 2),                                      # fp32, of 32
    ("f32", "same", [9000] + [700] * 3, [5] + [700] * 3, 32, 32, 136, 128, 0),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", LONG, ids=lambda c: f"{c[0]}-{c[1]}-{c[6]}-{c[8]}")
def test_a_long_sequence_among_many_rows(atp, case, causal):
    """More new rows than the call wants items for, and a sequence or two of thousands of keys: those keys are cut.  Three heads and a few sequences are
    compared with the oracle, every row is finite, a second call gives the same bits."""
    dtype, kind, lengths, new, heads, hk, d, page, max_new = case
    print(f"long {case[:2]} {case[4:]} {causal}", flush=True)
    rng = np.random.default_rng(72)
    p = Pages(atp, rng, lengths, hk, d, page, dtype, kind, most=-(-max(lengths) // page) + 3, fill=False)
    n = sum(lengths)
    K, V = (torch.randn((n, hk, d), generator=torch.Generator("cuda").manual_seed(s), device="cuda").to(TORCH[dtype]) for s in (1, 2))
    of_keys = offsets_of(lengths)
    table, length = ints(p.table), ints(lengths)
    atp.cache_write(p.cache, K, V, table, length, ints(of_keys))
    if kind == "e4m3":
        K, V = atp.cache_read(p.cache, table, length, ints(of_keys), tokens=n, dtype=torch.float32)
    offs = offsets_of(new)
    Q = randn(rng, (sum(new) + 1, heads, d), dtype, 2.0)
    out = torch.full_like(Q, 7.0)
    ws = torch.full((atp.attention_paged_workspace(p.cache, len(lengths), p.table.shape[1], sum(new) + 1, heads, TORCH[dtype], max_new),), 255, dtype=torch.uint8, device="cuda")
    call = lambda out: atp.attention_paged(Q, p.cache, table, length, ints(offs), causal=causal, max_new=max_new, workspace=ws, out=out)  # noqa: E731
    got = call(out)
    torch.cuda.synchronize()
    assert torch.isfinite(got.float()).all() and (got[sum(new):] == 7.0).all()
    assert torch.equal(call(torch.full_like(Q, 7.0)), got)
    some = sorted({*np.argsort(lengths)[-2:].tolist(), 0, len(lengths) // 2, len(lengths) - 1})
    for s in some:
        rows, keys = slice(offs[s], min(offs[s + 1], offs[s] + 20)), slice(of_keys[s], of_keys[s + 1])
        m = rows.stop - rows.start
        held = lengths[s] - (new[s] - m)   # (the first rows of the sequence: as if the later ones were not there yet)
        for h in (0, heads // 2 + 1, heads - 1):
            one = lambda x, at: [host(x[keys, at:at + 1])[:held if causal else None]]  # noqa: E731
            want = so.attention(host(Q[rows, h:h + 1]), one(K, h * hk // heads), one(V, h * hk // heads), [0, m], [held], causal, 0.0)
            check(host(got[rows, h:h + 1]), *want, dtype, lengths[s])


def test_a_long_sequence_among_many_rows_takes_no_longer_than_by_itself(atp):
    """8 chunks of 512 tokens and one token over 65536 keys: together no more than three times what the two take one after the other."""
    heads, hk, d, page = 32, 8, 128, 64

    def call(lengths, new):
        held = np.array(lengths) // page
        cache = atp.PagedCache.empty(int(held.sum()), hk, page, d, torch.bfloat16)
        table = np.full((len(lengths), 65536 // page), -1)
        for s, h in enumerate(held):
            table[s, :h] = held[:s].sum() + np.arange(h)
        Q, args = torch.ones((sum(new), heads, d), dtype=torch.bfloat16, device="cuda"), (ints(table), ints(lengths), ints(offsets_of(new)))
        out = torch.zeros_like(Q)
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        took = []
        for _ in range(6):
            start.record()
            atp.attention_paged(Q, cache, *args, max_new=max(new), out=out)
            end.record()
            torch.cuda.synchronize()
            took.append(start.elapsed_time(end) * 1e3)
        return min(took)

    chunks, single, both = call([512] * 8, [512] * 8), call([65536], [1]), call([512] * 8 + [65536], [512] * 8 + [1])
    print(f"chunks {chunks:.0f} us, single {single:.0f}, together {both:.0f}", flush=True)
    assert both <= 3 * (chunks + single)


# ------------------------------------------------------------------ every code under every exponent
def _all_codes(atp, page):
    """A cache of one head of 256 features with the codes 0 to 255 under each of the exponents 0 to 254, a position an exponent; and what they stand for."""
    cache = atp.PagedCache.empty(256 // page, 1, page, 256, torch.float8_e4m3fn)
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    byte = torch.arange(256).clamp(max=254)   # (the last position repeats the last exponent)
    for pages, scale in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)):
        pages.view(torch.uint8).copy_(codes.expand(pages.shape))
        scale.copy_(byte.view(scale.shape))
    return cache, codes.view(torch.float8_e4m3fn).double().numpy()[None] * np.exp2(byte.double().numpy() - 127)[:, None]


def _rounded(exact, dtype):
    """Nearest value of the type, ties to even, infinity where that is 2^128 (an intermediate rounding to fp32 is none: codes have four bits)."""
    return torch.from_numpy(exact).float().to(TORCH[dtype]).double().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_under_every_exponent_is_read_as_the_nearest_value(atp, dtype):
    """Exact from the smallest step of the type on; 2^128 and above are infinite, and what lies below bf16's smallest step is rounded to it or to zero."""
    cache, exact = _all_codes(atp, 16)
    K, V = atp.cache_read(cache, ints(np.arange(16)[None]), ints([256]), ints([0, 256]), tokens=256, dtype=TORCH[dtype])
    want = _rounded(exact, dtype)
    for got in (K, V):
        assert np.array_equal(host(got)[:, 0], want, equal_nan=True)
    step = 2.0 ** (-133 if dtype == "bf16" else -149)
    inside = (np.abs(exact) < 2.0 ** 128) & (exact % step == 0)
    assert np.array_equal(want[inside], exact[inside]) and np.isinf(want[np.abs(exact) >= 2.0 ** 128]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 200])
def test_every_code_under_every_exponent_is_attended_as_its_value(atp, dtype, rows):
    """One key a sequence: its weight is 1, so O is what reading gives, not finite where that is not.  The key itself is zeros: under the last exponents its score
    would be infinite or NaN."""
    cache, exact = _all_codes(atp, 1)
    cache.K.view(torch.uint8).zero_()
    Q = torch.zeros((256 * rows, 1, 256), dtype=TORCH[dtype], device="cuda")
    got = atp.attention_paged(Q, cache, ints(np.arange(256)[:, None]), ints([1] * 256), ints(rows * np.arange(257)), causal=False, max_new=rows)
    got = host(got).reshape(256, rows, 256)
    want = _rounded(exact, dtype)
    fine = np.isfinite(want)
    for r in (0, rows - 1):
        assert np.array_equal(got[:, r][fine], want[fine]) and not np.isfinite(got[:, r][~fine]).any()


# ------------------------------------------------------------------ values that are not finite where keys are cut
SPOILT = [
    # dtype, cache, lengths, new tokens, heads, kv_heads, d_h, page size, spoilt positions of the sequences
    ("bf16", "same", [3000, 700], [200, 150], 4, 1, 64, 64, [[2850, 2910, 2999], [600]]),       # row tiles of 128
    ("bf16", "same", [3000, 700], [200, 150], 4, 1, 80, 16, [[2850, 2910, 2999], [600]]),
    ("bf16", "e4m3", [3000, 700], [200, 150], 2, 1, 128, 64, [[2850, 2910, 2999], [600]]),
    ("bf16", "e4m3", [2000], [130], 2, 2, 256, 32, [[1900, 1999]]),
    ("bf16", "same", [4000, 900], [20, 7], 3, 1, 128, 64, [[3985, 3999], [896]]),               # of 32
    ("bf16", "same", [4000, 900], [20, 7], 3, 1, 72, 16, [[3985, 3999], [896]]),
    ("bf16", "e4m3", [4000, 900], [20, 7], 3, 1, 64, 32, [[3985, 3999], [896]]),
    ("f32", "same", [2000, 700], [100, 90], 2, 1, 64, 16, [[1930, 1999], [650]]),               # fp32, of 128
    ("f32", "e4m3", [2000, 700], [100, 90], 2, 1, 128, 64, [[1930, 1999], [650]]),
    ("f32", "same", [1500], [20], 2, 1, 200, 64, [[1485, 1499]]),
    ("f32", "same", [3000, 600], [10, 5], 2, 1, 64, 64, [[2993, 2999], [597]]),                 # of 32
    ("f32", "e4m3", [3000, 600], [10, 5], 2, 1, 128, 16, [[2993, 2999], [597]]),
]


@pytest.mark.parametrize("case", SPOILT, ids=lambda c: f"{c[0]}-{c[1]}-{c[3][0]}-{c[6]}")
def test_masked_values_that_are_not_finite_where_keys_are_cut(atp, case):
    """Sequences long enough to be cut, values spoilt (NaN in 8 bits, else infinite) at positions that some of the new tokens see: those before do not
    notice, the others not in the other features."""
    dtype, kind, lengths, new, heads, hk, d, page, spoilt = case
    print(f"spoilt {case[:2]} {case[2:8]}", flush=True)
    rng = np.random.default_rng(73)
    p = Pages(atp, rng, lengths, hk, d, page, dtype, kind)
    offs, hit = offsets_of(new), np.zeros(sum(new), bool)
    for s, positions in enumerate(spoilt):
        for at in positions:
            no, slot = so.place(p.table[s], at, page, p.n_pages)
            x = p.cache.V[no].float()
            x[:, slot, 3] = float("nan") if kind == "e4m3" else float("inf")
            p.cache.V[no] = x.to(p.cache.V.dtype)
        hit[offs[s]:offs[s + 1]] = np.arange(lengths[s] - new[s], lengths[s]) >= min(positions)
    assert hit.any() and not hit.all()
    assert atp.attention_paged_workspace(p.cache, len(lengths), p.table.shape[1], sum(new), heads, TORCH[dtype]) > 0   # (keys may be cut)
    Q = randn(rng, (sum(new), heads, d), dtype, 2.0)
    K, V, present = p.gathered()
    with np.errstate(invalid="ignore"):
        want = so.attention(host(Q), K, V, offs, lengths, True, 0.0, present)
    got = host(atp.attention_paged(Q, p.cache, ints(p.table), ints(lengths), ints(offs), max_new=max(new)))
    check(got[~hit], *(x[~hit] for x in want), dtype, max(lengths))
    rest = np.arange(d) != 3
    check(got[..., rest], want[0][..., rest], want[1][..., rest], want[2], want[3], dtype, max(lengths))
    assert not np.isfinite(got[hit][..., 3]).any()


def test_a_value_that_is_not_finite_costs_its_key_tile(atp):
    """In a prompt of 6000 tokens what it costs in one of 192, by the keys that are added row by row.  The value stands 64 tokens from the end, in the key tile
    5888 to 5951 (128 to 191), which the row tile 5888 to 5999 (128 to 191) crosses: of its 112 (64) rows the first 64 see 1 to 64 keys of the tile, 2080 in all,
    and the other 48 (none) all 64, so 5152 / 2080 = 2.48 times as many.  Twice that is allowed, for the noise of short times."""
    rng = np.random.default_rng(74)

    def took(n, spoilt):
        Q, K, V = (randn(rng, (n, 2, 128), "bf16") for _ in range(3))
        V[n - 64, :, 7] = float("inf") if spoilt else 1.0
        offs, out, times = ints([0, n]), torch.zeros_like(Q), []
        for _ in range(8):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            atp.attention_packed(Q, K, V, offs, out=out)
            end.record()
            torch.cuda.synchronize()
            times.append(start.elapsed_time(end) * 1e3)
        return min(times)

    clean, spoilt, short = took(6000, False), took(6000, True), took(192, True)
    print(f"6000 tokens {clean:.0f} us, spoilt {spoilt:.0f}, 192 spoilt {short:.0f}", flush=True)
    assert spoilt <= clean + 2 * 2.48 * short


# ------------------------------------------------------------------ very many sequences
def _single_keys(atp, rng, n_seq, long, most_new, dtype, kind, page):
    """n_seq sequences of one key, those in `long` {sequence: length} longer; pages in order.  -> (cache, lengths, first page of each)"""
    lengths = np.ones(n_seq, np.int64)
    for s, n in long.items():
        lengths[s] = n
    held = -(-lengths // page)
    first = np.concatenate([[0], np.cumsum(held)])
    cache = atp.PagedCache.empty(int(first[-1]), 1, page, 64, torch.float8_e4m3fn if kind == "e4m3" else TORCH[dtype])
    for x, seed in ((cache.K, 3), (cache.V, 4)):
        x.copy_(torch.randn(x.shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda"))
    if kind == "e4m3":
        cache.K_scale.fill_(127)
        cache.V_scale.fill_(126)
    table = first[:-1, None] + np.arange(held.max())
    table[np.arange(held.max())[None] >= held[:, None]] = -1
    return cache, lengths, first, ints(table)


def _check_single_keys(atp, Q, got, cache, lengths, first, offs, some, dtype):
    """Sequences of one key give its value, those in `some` what the oracle says."""
    f = 0.5 if cache.e4m3 else 1.0
    page = cache.page_size
    for s in some:
        rows = slice(offs[s], offs[s + 1])
        k, v = (host(x[first[s]:first[s + 1], 0].reshape(-1, 1, 64)[:lengths[s]]) for x in (cache.K, cache.V))
        check(host(got[rows]), *so.attention(host(Q[rows]), [k], [v * f], [0, rows.stop - rows.start], [int(lengths[s])], True, 0.0), dtype, int(lengths[s]))
    one = torch.ones(len(lengths), dtype=torch.bool)
    one[list(some)] = False
    new = np.diff(offs)
    one &= torch.from_numpy(new == 1)
    at = one.nonzero()[:, 0]
    value = cache.V.float().view(-1, page, 64)[torch.from_numpy(first[:-1])[at].cuda(), 0] * f
    assert torch.equal(got[torch.from_numpy(offs[:-1])[at].cuda()].float(), value[:, None].expand(-1, Q.shape[1], -1).to(TORCH[dtype]).float())


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same")])
def test_thousands_of_sequences_with_long_ones_at_the_end(atp, dtype, kind):
    """5000 single tokens, a few of them over thousands of keys and late: more than one step of the count within a lane's block, and keys are cut."""
    rng = np.random.default_rng(75)
    long = {4300: 1000, 4864: 3000, 4930: 700, 4999: 2500}
    cache, lengths, first, table = _single_keys(atp, rng, 5000, long, 1, dtype, kind, 32)
    new = np.ones(5000, np.int64)
    new[4864] = 9
    offs = offsets_of(new)
    assert atp.attention_paged_workspace(cache, 5000, table.shape[1], int(offs[-1]), 2, TORCH[dtype], 9) > 0
    Q = randn(rng, (int(offs[-1]), 2, 64), dtype, 2.0)
    for max_new in (0, 9):
        got = atp.attention_paged(Q, cache, table, ints(lengths), ints(offs), max_new=max_new)
        _check_single_keys(atp, Q, got, cache, lengths, first, offs, long, dtype)


@pytest.mark.parametrize("tokens", ["all", "few"])
def test_as_many_sequences_as_a_call_takes(atp, tokens):
    """65536 sequences, three of them long: a new token each (more rows than the chip wants), or new tokens for those three and two others only."""
    rng = np.random.default_rng(76)
    n_seq, long = 65536, {0: 9000, 40000: 5000, 65535: 8500}
    cache, lengths, first, table = _single_keys(atp, rng, n_seq, long, 1, "bf16", "same", 64)
    new = np.ones(n_seq, np.int64)
    if tokens == "few":
        new[:] = 0
        new[[0, 1023, 1024, 40000, 65535]] = 5, 1, 1, 1, 3
    offs = offsets_of(new)
    Q = randn(rng, (int(offs[-1]), 1, 64), "bf16", 2.0)
    print(f"65536 sequences, {tokens}", flush=True)
    args = (table, ints(lengths), ints(offs))
    got = atp.attention_paged(Q, cache, *args, max_new=5)
    torch.cuda.synchronize()
    _check_single_keys(atp, Q, got, cache, lengths, first, offs, long, "bf16")
    K, V = atp.cache_read(cache, *args, tokens=int(offs[-1]))
    s = torch.from_numpy(np.repeat(np.arange(n_seq), new))
    at = torch.from_numpy(lengths[s.numpy()] - new[s.numpy()] + np.arange(int(offs[-1])) - offs[s.numpy()])
    where = torch.from_numpy(first[s.numpy()]) + at // 64
    assert torch.equal(K[:, 0], cache.K[where.cuda(), 0, (at % 64).cuda()]) and torch.equal(V[:, 0], cache.V[where.cuda(), 0, (at % 64).cuda()])
    atp.cache_write(cache, K.flip(0), V.flip(0), *args)
    assert torch.equal(cache.K[where.cuda(), 0, (at % 64).cuda()], K[:, 0].flip(0)) and torch.equal(cache.V[where.cuda(), 0, (at % 64).cuda()], V[:, 0].flip(0))
    # packed: a token each
    x = [randn(rng, (n_seq, 1, 64), "bf16") for _ in range(3)]
    assert tokens == "few" or torch.equal(atp.attention_packed(*x, ints(np.arange(n_seq + 1))), x[2])
