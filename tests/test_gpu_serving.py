"""Packed and paged attention, writing and reading a paged cache: GPU against the float64 oracle on the inputs that the GPU holds.

Tolerances are bounds for each element, from the roundings that the definition cannot avoid: with p the softmax weights and A = Σ p·|v|,
  |O − ref| <= h·|O| + A·(4·δ + 2·(n + 16)·2^-24 + w),
h: half a step of the storage type (2^-8 bf16, 2^-24 fp32); w: a rounding of the weights to the type of the matrix product (2^-8, 0);
δ: error of a score, d_h + 4 fp32 roundings of sums up to Σ|q·k| and two of the score itself before its exponential; n: terms of the fp32
sums (a weight carries the error of its own score and of the running maximum's, numerator and denominator each: factor 4).
Codes of 8 bits, exponents and rows that are only moved are compared bit by bit."""
import numpy as np
import pytest
import torch

from oracle import serving as so

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def atp():
    import paper_2403_02352_amd as m
    return m


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def randn(rng, shape, dtype, scale=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(TORCH[dtype]).cuda()


def tolerance(dtype, ref, A, reach, top, n, d):
    delta = reach * (d + 4) * 2.0 ** -24 + top * 2.0 ** -22
    rel = 4 * delta[..., None] + 2 * (n + 16) * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    return HALF[dtype] * np.abs(ref) + A * rel + 1e-37


def check(got, ref, A, reach, top, dtype, n):
    """Rows outside every sequence are NaN in ref and looked at elsewhere."""
    inside = ~np.isnan(ref).all(-1)
    assert np.isfinite(got[inside]).all()
    off = np.abs(got - ref)[inside]
    tol = tolerance(dtype, ref, A, reach, top, n, ref.shape[-1])[inside]
    worst = (off / tol).max() if off.size else 0.0
    print(f"  worst {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0


def offsets_of(lengths, first=0):
    return np.concatenate([[0], np.cumsum(lengths)]) + first


# ------------------------------------------------------------------ packed prompts
PACKED = [
    # lengths, heads, kv_heads, d_h
    ([1], 1, 1, 64),
    ([5, 0, 1, 33], 4, 2, 64),          # an empty sequence, one of a single token
    ([64, 65, 63], 2, 2, 128),          # around a tile of keys
    ([127, 128, 129], 3, 1, 64),        # around a tile of queries, three heads to a key head
    ([300, 7], 8, 1, 128),              # eight heads to a key head
    ([40, 90], 7, 7, 32),               # narrow heads, an odd number of them
    ([70, 20], 2, 1, 80),               # widths that are no power of two
    ([50, 33], 2, 2, 96),
    ([140, 3], 2, 1, 256),
    ([17] * 70, 2, 1, 64),              # more sequences than a wave has lanes
    ([700], 2, 1, 128),
    ([90, 31], 2, 1, 8),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", PACKED, ids=str)
def test_attention_packed(atp, dtype, causal, case):
    lengths, heads, hk, d = case
    rng = np.random.default_rng(11)
    tokens = sum(lengths) + 3   # three rows behind the last sequence
    print(f"packed {dtype} {causal} {case}", flush=True)
    qkv = randn(rng, (tokens, heads + 2 * hk, d), dtype)
    qkv[:, :heads] *= 2
    qkv[sum(lengths):] = float("nan")   # what lies there reaches nobody
    Q, K, V = qkv[:, :heads], qkv[:, heads:heads + hk], qkv[:, heads + hk:]
    offs = offsets_of(lengths)
    out = torch.full((tokens, heads, d), 7.0, dtype=TORCH[dtype], device="cuda")
    got = atp.attention_packed(Q, K, V, ints(offs), causal=causal, out=out)
    torch.cuda.synchronize()
    k, v = host(K), host(V)
    cut = lambda x: [x[a:a + n] for a, n in so.bounds(offs, tokens)]  # noqa: E731
    check(host(got), *so.attention(host(Q), cut(k), cut(v), offs, lengths, causal, 0.0), dtype, max(lengths))
    assert (got[sum(lengths):] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_packed_rows_before_the_first_sequence_stay(atp, dtype):
    rng = np.random.default_rng(12)
    lengths, heads, hk, d = [20, 50], 2, 1, 64
    offs = offsets_of(lengths, 9)
    Q, K, V = randn(rng, (90, heads, d), dtype), randn(rng, (90, hk, d), dtype), randn(rng, (90, hk, d), dtype)
    out = torch.full_like(Q, 5.0)
    atp.attention_packed(Q, K, V, ints(offs), out=out)
    k, v = host(K), host(V)
    cut = lambda x: [x[a:a + n] for a, n in so.bounds(offs, 90)]  # noqa: E731
    check(host(out), *so.attention(host(Q), cut(k), cut(v), offs, lengths, True, 0.0), dtype, 50)
    assert (out[:9] == 5.0).all() and (out[79:] == 5.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("what", ["K", "V"])
def test_attention_packed_masked_values_that_are_not_finite(atp, dtype, bad, what):
    """Row j of K or V spoilt: queries before j, and the other sequences, do not notice."""
    rng = np.random.default_rng(13)
    lengths, heads, hk, d = [200, 45, 150], 4, 2, 64
    offs = offsets_of(lengths)
    tokens = sum(lengths)
    Q, K, V = randn(rng, (tokens, heads, d), dtype, 2.0), randn(rng, (tokens, hk, d), dtype), randn(rng, (tokens, hk, d), dtype)
    spoilt = {"K": K, "V": V}[what]
    for t in (70, 130, 199, 200 + 44, 245 + 149):
        spoilt[t, :, 5] = bad
    got = host(atp.attention_packed(Q, K, V, ints(offs)))
    k, v = host(K), host(V)
    cut = lambda x: [x[a:a + n] for a, n in so.bounds(offs, tokens)]  # noqa: E731
    with np.errstate(invalid="ignore"):
        ref, A, reach, top = so.attention(host(Q), cut(k), cut(v), offs, lengths, True, 0.0)
    before = np.zeros(tokens, dtype=bool)
    for a, first_bad in ((0, 70), (200, 44), (245, 149)):
        before[a:a + first_bad] = True
    check(got[before], ref[before], A[before], reach[before], top[before], dtype, 200)
    # feature by feature where values are spoilt: the others of a row that sees it are as they should be
    if what == "V":
        rest = np.arange(d) != 5
        seen = ~before
        check(got[seen][..., rest], ref[seen][..., rest], A[seen][..., rest], reach[seen], top[seen], dtype, 200)
        assert not np.isfinite(got[seen][..., 5]).any()
    elif bad != bad:
        assert np.isnan(got[~before]).all()


def test_attention_packed_scores_of_minus_infinity(atp):
    """A query all of whose scores are -inf gives zeros; single keys at -inf weigh nothing."""
    for dtype in ("bf16", "f32"):
        Q = torch.ones((80, 1, 64), dtype=TORCH[dtype], device="cuda")
        K = torch.zeros((80, 1, 64), dtype=TORCH[dtype], device="cuda")
        V = torch.ones((80, 1, 64), dtype=TORCH[dtype], device="cuda")
        K[:3, :, 0] = float("-inf")
        K[40, :, 0] = float("-inf")
        V[40] = 9.0
        got = host(atp.attention_packed(Q, K, V, ints([0, 80])))
        assert (got[:3] == 0).all() and (np.abs(got[3:] - 1.0) <= HALF[dtype] * 4).all()


# ------------------------------------------------------------------ a paged cache
class Pages:
    """A cache on the GPU with its host copy; the table is a permutation of the pages."""

    def __init__(self, atp, rng, lengths, hk, d, page, dtype, kind, spare=2, most=None, fill=True):
        held = [-(-max(n, 0) // page) for n in lengths]
        n_pages = sum(held) + spare
        self.page, self.n_pages, self.lengths = page, n_pages, lengths
        order = rng.permutation(n_pages)
        most = max(held + [1]) if most is None else most
        self.table = np.full((len(lengths), most), -1)
        at = 0
        for s, h in enumerate(held):
            self.table[s, :h] = order[at:at + h]
            at += h
        self.cache = atp.PagedCache.empty(n_pages, hk, page, d, torch.float8_e4m3fn if kind == "e4m3" else TORCH[dtype])
        if fill:
            for pages, scale in ((self.cache.K, self.cache.K_scale), (self.cache.V, self.cache.V_scale)):
                x = rng.standard_normal((n_pages, hk, page, d)) * np.exp(rng.standard_normal((n_pages, hk, page, 1)) * 0.5)
                if scale is None:
                    pages.copy_(torch.from_numpy(x))
                else:
                    codes, e = so.quantise_rows(x)
                    pages.copy_(torch.from_numpy(codes).float().to(torch.float8_e4m3fn))
                    scale.copy_(torch.from_numpy(e))

    def pages(self):
        """(K pages, K exponents, V pages, V exponents) on the host."""
        c = self.cache
        n = lambda s: None if s is None else s.cpu().numpy()  # noqa: E731
        return host(c.K), n(c.K_scale), host(c.V), n(c.V_scale)

    def gathered(self):
        k, ks, v, vs = self.pages()
        K = [so.gather(k, ks, self.table[s], n) for s, n in enumerate(self.lengths)]
        V = [so.gather(v, vs, self.table[s], n) for s, n in enumerate(self.lengths)]
        return [x[0] for x in K], [x[0] for x in V], [x[1] for x in K]


PAGED = [
    # lengths, new tokens, heads, kv_heads, d_h, page size
    ([1], [1], 1, 1, 64, 16),
    ([500, 3, 77], [1, 1, 1], 4, 1, 128, 16),           # a step of decoding
    ([0, 40, 1], [1, 1, 1], 8, 2, 64, 32),              # a new token with no key at all
    ([200, 90, 64], [70, 5, 0], 4, 2, 64, 64),          # chunks, one sequence without any
    ([30, 10], [50, 10], 2, 1, 128, 8),                 # more new tokens than positions: the first see nothing
    ([129, 128, 127], [129, 128, 127], 2, 2, 128, 128),  # whole prompts
    ([333, 61], [3, 40], 14, 2, 80, 16),
    ([100, 45], [9, 45], 3, 3, 96, 256),                # pages longer than the sequences
    ([90, 33], [2, 33], 6, 2, 256, 1),                  # pages of a single position
    ([40] * 70, [1] * 70, 2, 1, 64, 16),
    ([2500, 9], [1, 1], 32, 4, 128, 64),                # long enough to be split
    ([1800], [64], 4, 1, 64, 32),
    ([64, 50], [2, 1], 2, 2, 8, 16),
]


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", PAGED, ids=lambda c: str(c)[:60])
def test_attention_paged(atp, dtype, kind, causal, case):
    lengths, new, heads, hk, d, page = case
    print(f"paged {dtype} {kind} {causal} {str(case)[:80]}", flush=True)
    rng = np.random.default_rng(21)
    p = Pages(atp, rng, lengths, hk, d, page, dtype, kind)
    tokens = sum(new) + 2
    Q = randn(rng, (tokens, heads, d), dtype, 2.0)
    offs = offsets_of(new)
    K, V, present = p.gathered()
    want = so.attention(host(Q), K, V, offs, lengths, causal, 0.0, present)
    for max_new in (0, max(new), 1):   # a hint only
        out = torch.full((tokens, heads, d), 7.0, dtype=TORCH[dtype], device="cuda")
        got = atp.attention_paged(Q, p.cache, ints(p.table), ints(lengths), ints(offs), causal=causal, max_new=max_new, out=out)
        torch.cuda.synchronize()
        check(host(got), *want, dtype, max(lengths))
        assert (got[sum(new):] == 7.0).all()


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
def test_attention_paged_pages_that_are_not_there(atp, dtype, kind):
    """Page numbers outside the cache hold no keys, wherever they stand; the spare pages hold NaN."""
    rng = np.random.default_rng(22)
    lengths, new, heads, hk, d, page = [300, 200, 100], [1, 30, 100], 4, 2, 64, 16
    p = Pages(atp, rng, lengths, hk, d, page, dtype, kind)
    p.table[0, [0, 7, 18]] = [-1, p.n_pages, -2 ** 31]
    p.table[1, :] = -1
    p.table[2, 6] = 2 ** 31 - 1
    spare = sorted(set(range(p.n_pages)) - set(p.table.ravel().tolist()))
    assert spare
    p.cache.K[spare] = torch.full_like(p.cache.K[spare].float(), float("nan")).to(p.cache.K.dtype)
    p.cache.V[spare] = torch.full_like(p.cache.V[spare].float(), float("nan")).to(p.cache.V.dtype)
    Q = randn(rng, (sum(new), heads, d), dtype, 2.0)
    offs = offsets_of(new)
    K, V, present = p.gathered()
    for causal in (True, False):
        got = host(atp.attention_paged(Q, p.cache, ints(p.table), ints(lengths), ints(offs), causal=causal))
        check(got, *so.attention(host(Q), K, V, offs, lengths, causal, 0.0, present), dtype, 300)
        assert (got[1:31] == 0).all()   # nothing is seen there


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_paged_lengths_beyond_the_table(atp, dtype):
    """Positions that the table does not reach hold no keys; a negative length is an empty sequence."""
    rng = np.random.default_rng(23)
    p = Pages(atp, rng, [64, 64, 64], 1, 64, 16, dtype, "same")
    lengths, new = [70, -5, 64], [10, 2, 1]
    p.lengths = lengths
    Q = randn(rng, (13, 2, 64), dtype)
    offs = offsets_of(new)
    K, V, present = p.gathered()
    got = host(atp.attention_paged(Q, p.cache, ints(p.table), ints(lengths), ints(offs)))
    check(got, *so.attention(host(Q), K, V, offs, [70, 0, 64], True, 0.0, present), dtype, 70)
    assert (got[10:12] == 0).all()


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
def test_attention_paged_masked_values_that_are_not_finite(atp, dtype, kind):
    rng = np.random.default_rng(24)
    lengths, new, heads, hk, d, page = [130], [100], 2, 1, 64, 16
    p = Pages(atp, rng, lengths, hk, d, page, dtype, kind)
    for pos in (90, 120, 129):
        page_no, slot = so.place(p.table[0], pos, page, p.n_pages)
        x = p.cache.V[page_no].float()
        x[:, slot, 3] = float("nan") if kind == "e4m3" else float("inf")
        p.cache.V[page_no] = x.to(p.cache.V.dtype)
    # positions behind the length, in the last page
    page_no, _ = so.place(p.table[0], 129, page, p.n_pages)
    for t in (p.cache.K, p.cache.V):
        x = t[page_no].float()
        x[:, 2:] = float("nan")
        t[page_no] = x.to(t.dtype)
    Q = randn(rng, (100, heads, d), dtype, 2.0)
    K, V, present = p.gathered()
    got = host(atp.attention_paged(Q, p.cache, ints(p.table), ints(lengths), ints([0, 100])))
    with np.errstate(invalid="ignore"):
        ref, A, reach, top = so.attention(host(Q), K, V, [0, 100], lengths, True, 0.0, present)
    before = np.arange(100) + 30 < 90
    check(got[before], ref[before], A[before], reach[before], top[before], dtype, 130)
    rest = np.arange(d) != 3
    check(got[..., rest], ref[..., rest], A[..., rest], reach, top, dtype, 130)
    assert not np.isfinite(got[~before][..., 3]).any()


# ------------------------------------------------------------------ writing and reading
ROWS = [
    # lengths, new tokens, kv_heads, d_h, page size
    ([1], [1], 1, 64, 16),
    ([5, 0, 300, 40], [5, 1, 130, 0], 2, 64, 16),
    ([33, 64], [40, 1], 8, 128, 64),            # more new tokens than positions
    ([20, 90], [20, 3], 3, 80, 32),
    ([50] * 130, [2] * 130, 1, 8, 8),           # more sequences than two waves have lanes
    ([77, 10], [30, 10], 5, 256, 1),
    ([40], [40], 2, 96, 1024),
]


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
@pytest.mark.parametrize("case", ROWS, ids=lambda c: str(c)[:60])
def test_cache_write_and_read(atp, dtype, kind, case):
    lengths, new, hk, d, page = case
    print(f"rows {dtype} {kind} {str(case)[:80]}", flush=True)
    rng = np.random.default_rng(31)
    p = Pages(atp, rng, lengths, hk, d, page, dtype, kind)
    p.table[0, 0] = -1 if len(lengths) > 1 else p.table[0, 0]   # a page that is not there
    tokens = sum(new) + 2
    kv = (randn(rng, (tokens, 2 * hk, d), dtype) * torch.from_numpy(np.exp2(rng.integers(-30, 30, (tokens, 2 * hk, 1)))).cuda()).to(TORCH[dtype])
    K, V = kv[:, :hk], kv[:, hk:]
    K[0, 0, 1], V[0, 0, 2] = float("nan"), float("-inf")
    K[tokens - 3], V[tokens - 3] = 0.0, 448.0 * 2.0 ** -3
    offs = offsets_of(new)
    before = p.pages()
    atp.cache_write(p.cache, K, V, ints(p.table), ints(lengths), ints(offs))
    torch.cuda.synchronize()
    after = p.pages()
    places = so.new_places(p.table, lengths, offs, tokens, page, p.n_pages)
    for x, (pages, scale), (had, had_scale) in ((host(K), after[:2], before[:2]), (host(V), after[2:], before[2:])):
        want, want_scale = had.copy(), None if scale is None else had_scale.copy()
        codes, e = so.quantise_rows(x) if kind == "e4m3" else (x, None)
        for t, pg, slot in places:
            want[pg, :, slot] = codes[t]
            if scale is not None:
                want_scale[pg, :, slot] = e[t]
        assert np.array_equal(pages, want, equal_nan=True)
        assert scale is None or np.array_equal(scale, want_scale)
    # and back, into column blocks of a wider matrix
    out = torch.full((tokens, 2 * hk + 1, d), 3.0, dtype=TORCH[dtype], device="cuda")
    Ko, Vo = atp.cache_read(p.cache, ints(p.table), ints(lengths), ints(offs), out=(out[:, :hk], out[:, hk + 1:]))
    torch.cuda.synchronize()
    for got, pages, scale in ((Ko, *after[:2]), (Vo, *after[2:])):
        want = np.full((tokens, hk, d), 3.0)
        want[:sum(new)] = 0.0
        for t, pg, slot in places:
            want[t] = pages[pg, :, slot] if scale is None else so.dequantise_rows(pages[pg, :, slot], scale[pg, :, slot])
        assert np.array_equal(host(got), want, equal_nan=True)
    assert (out[:, hk] == 3.0).all()


def test_quantised_rows_at_the_ends_of_the_range(atp):
    """Powers of two from the smallest exponent to the largest value, amounts on both sides of a power's limit, subnormal rows."""
    for dtype in ("bf16", "f32"):
        tops = [2.0 ** e for e in range(-149 if dtype == "f32" else -133, 128)] + [448.0 * 2.0 ** e for e in range(-130, 120, 7)]
        tops += [float(torch.nextafter(torch.tensor(448.0 * 2.0 ** e), torch.tensor(1e38))) for e in range(-100, 110, 9)] + [float(torch.finfo(TORCH[dtype]).max), 0.0]
        rng = np.random.default_rng(32)
        x = np.array(tops)[:, None] * np.concatenate([[1.0], rng.uniform(-1, 1, 15)])[None]
        K = torch.from_numpy(x).to(TORCH[dtype]).cuda().view(-1, 1, 16)
        n = K.shape[0]
        cache = atp.PagedCache.empty(-(-n // 16), 1, 16, 16, torch.float8_e4m3fn)
        table, length, offs = ints(np.arange(-(-n // 16))[None]), ints([n]), ints([0, n])
        atp.cache_write(cache, K, K, table, length, offs)
        codes, e = so.quantise_rows(host(K))
        assert np.array_equal(host(cache.K).reshape(-1, 16)[:n], codes[:, 0])
        assert np.array_equal(cache.K_scale.cpu().numpy().reshape(-1)[:n], e[:, 0])
        back, _ = atp.cache_read(cache, table, length, offs, out=(torch.empty_like(K), torch.empty_like(K)))
        want = torch.from_numpy(so.dequantise_rows(codes, e)).to(torch.float32).to(TORCH[dtype])
        assert torch.equal(back.cpu(), want)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
def test_prompts_then_steps(atp, dtype, kind):
    """Prompts through packed attention and into the cache, then a chunk and single tokens over the cache: every output is that of causal
    attention over all the keys and values the cache stands for; rotary positions from atp.rope."""
    rng = np.random.default_rng(41)
    heads, hk, d, page = 4, 2, 64, 16
    prompts, steps = [45, 1, 100], [[7, 1, 0], [1, 1, 1], [1, 1, 1]]
    total = [n + sum(s[i] for s in steps) for i, n in enumerate(prompts)]
    p = Pages(atp, rng, total, hk, d, page, dtype, kind, fill=False)
    table = ints(p.table)

    def rows(new, start):
        x = randn(rng, (sum(new), heads + 2 * hk, d), dtype)
        q, k, v = x[:, :heads], x[:, heads:heads + hk], x[:, heads + hk:]
        q, k = q.contiguous(), k.contiguous()
        at = 0
        for n, pos in zip(new, start):   # every sequence rotates from its own position
            if n:
                for y in (q, k):
                    y[at:at + n] = atp.rope(y[at:at + n].reshape(1, n, -1).contiguous(), y.shape[1], pos0=pos).view(n, y.shape[1], d)
            at += n
        return q, k, v

    q, k, v = rows(prompts, [0] * 3)
    offs = offsets_of(prompts)
    got = atp.attention_packed(q, k, v, ints(offs))
    cut = lambda x: [x[a:a + n] for a, n in so.bounds(offs, sum(prompts))]  # noqa: E731
    check(host(got), *so.attention(host(q), cut(host(k)), cut(host(v)), offs, prompts, True, 0.0), dtype, 100)
    atp.cache_write(p.cache, k, v, table, ints(prompts), ints(offs))
    if kind == "same":   # the same attention over the cache
        over = atp.attention_paged(q, p.cache, table, ints(prompts), ints(offs))
        check(host(over), *so.attention(host(q), cut(host(k)), cut(host(v)), offs, prompts, True, 0.0), dtype, 100)
    now = list(prompts)
    for new in steps:
        q, k, v = rows(new, now)
        now = [a + b for a, b in zip(now, new)]
        offs = offsets_of(new)
        atp.cache_write(p.cache, k, v, table, ints(now), ints(offs))
        got = atp.attention_paged(q, p.cache, table, ints(now), ints(offs), max_new=max(new))
        p.lengths = now
        K, V, present = p.gathered()
        check(host(got), *so.attention(host(q), K, V, offs, now, True, 0.0, present), dtype, max(now))
    back, _ = atp.cache_read(p.cache, table, ints(now), ints(offsets_of(now)), tokens=sum(now), dtype=TORCH[dtype])
    assert np.array_equal(host(back), np.concatenate(K))


def test_attention_paged_over_principal_keys(atp):
    """Without the mask and with r_s principal keys in the pages it is atp.attention with a rank for each sequence."""
    rng = np.random.default_rng(42)
    heads, d, ranks, L = 2, 64, [20, 33], 50
    p = Pages(atp, rng, ranks, heads, d, 16, "bf16", "same", fill=False)
    K, V, Q = (randn(rng, (n, heads, d), "bf16") for n in (sum(ranks), sum(ranks), 2 * L))
    offs = offsets_of(ranks)
    atp.cache_write(p.cache, K, V, ints(p.table), ints(ranks), ints(offs))
    got = atp.attention_paged(Q, p.cache, ints(p.table), ints(ranks), ints([0, L, 2 * L]), causal=False)
    for s, (a, r) in enumerate(so.bounds(offs, sum(ranks))):
        one = atp.attention(Q[s * L:(s + 1) * L].reshape(1, L, -1), K[a:a + r].reshape(1, r, -1), V[a:a + r].reshape(1, r, -1), heads)
        k, v = host(K[a:a + r]), host(V[a:a + r])
        ref, A, reach, top = so.attention(host(Q[s * L:(s + 1) * L]), [k], [v], [0, L], [r], False, 0.0)
        tol = tolerance("bf16", ref, A, reach, top, r, d)
        assert (np.abs(host(got[s * L:(s + 1) * L]) - host(one).reshape(L, heads, d)) <= 2 * tol).all()


# ------------------------------------------------------------------ streams, graphs, large caches
def test_calls_on_a_side_stream_and_twice_at_once(atp):
    """Two streams with workspaces and outputs of their own give what one gives."""
    rng = np.random.default_rng(51)
    lengths, heads, hk, d = [3000, 40], 8, 2, 128
    p = Pages(atp, rng, lengths, hk, d, 64, "bf16", "e4m3")
    table, length, offs = ints(p.table), ints(lengths), ints([0, 1, 2])
    Q = [randn(rng, (2, heads, d), "bf16") for _ in range(2)]
    want = [atp.attention_paged(q, p.cache, table, length, offs, max_new=1) for q in Q]
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for q, s in zip(Q, side):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(atp.attention_paged(q, p.cache, table, length, offs, max_new=1))
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind", ["same", "e4m3"])
def test_a_step_in_a_graph_follows_its_inputs(atp, kind):
    """Write and attend captured once; replays with other lengths, tokens and pages give what eager calls give."""
    rng = np.random.default_rng(52)
    heads, hk, d, page = 4, 2, 64, 16
    p = Pages(atp, rng, [2000, 600], hk, d, page, "bf16", kind)
    twin = Pages(atp, rng, [2000, 600], hk, d, page, "bf16", kind)
    x = randn(rng, (2, heads + 2 * hk, d), "bf16")
    table, length, offs = ints(p.table), ints([10, 10]), ints([0, 1, 2])
    out = torch.zeros((2, heads, d), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(256, atp.attention_paged_workspace(p.cache, 2, table.shape[1], 2, heads, torch.bfloat16, 1)), dtype=torch.uint8, device="cuda")

    def step(cache, out, ws):
        atp.cache_write(cache, x[:, heads:heads + hk], x[:, heads + hk:], table, length, offs)
        atp.attention_paged(x[:, :heads], cache, table, length, offs, max_new=1, workspace=ws, out=out)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(p.cache, out, ws)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(p.cache, out, ws)
    # (the run before the capture has written its tokens: the twin starts from there)
    for a, b in ((p.cache.K, twin.cache.K), (p.cache.V, twin.cache.V), (p.cache.K_scale, twin.cache.K_scale), (p.cache.V_scale, twin.cache.V_scale)):
        if a is not None:
            b.view(torch.uint8).copy_(a.view(torch.uint8))
    for n in ([2000, 600], [1, 1], [700, 599], [33, 0], [1999, 64]):
        length.copy_(ints(n))
        x.copy_(randn(rng, x.shape, "bf16"))
        if n[0] == 700:   # the sequences change places
            table.copy_(ints(p.table[::-1].copy()))
            length.copy_(ints([599, 700]))
        if n[0] == 33:
            offs.copy_(ints([0, 2, 2]))
        graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros_like(out)
        step(twin.cache, want, None)
        torch.cuda.synchronize()
        assert torch.equal(out, want), n
        assert torch.equal(p.cache.K.view(torch.uint8), twin.cache.K.view(torch.uint8))


def test_same_inputs_give_the_same_bits(atp):
    rng = np.random.default_rng(53)
    p = Pages(atp, rng, [5000, 900, 33], 2, 128, 64, "bf16", "same")
    Q = randn(rng, (40, 8, 128), "bf16")
    args = (ints(p.table), ints([5000, 900, 33]), ints([0, 1, 36, 40]))
    first = atp.attention_paged(Q, p.cache, *args)
    for _ in range(5):
        assert torch.equal(atp.attention_paged(Q, p.cache, *args), first)


def test_a_cache_beyond_32_bit_offsets(atp):
    """Pages that start behind 2^32 bytes and 2^31 elements are written, read and attended."""
    rng = np.random.default_rng(54)
    hk, d, page = 8, 128, 64
    n_pages = 2 ** 31 // (hk * d * page) + 300   # 4.04 GiB of bf16 each for keys and values
    cache = atp.PagedCache.empty(n_pages, hk, page, d, torch.bfloat16)
    table = np.array([[n_pages - 1, 0, n_pages - 2]])
    K, V, Q = randn(rng, (150, hk, d), "bf16"), randn(rng, (150, hk, d), "bf16"), randn(rng, (150, hk, d), "bf16", 2.0)
    args = (ints(table), ints([150]), ints([0, 150]))
    atp.cache_write(cache, K, V, *args)
    Ko, Vo = atp.cache_read(cache, *args, tokens=150)
    assert torch.equal(Ko, K) and torch.equal(Vo, V)
    got = host(atp.attention_paged(Q, cache, *args))
    check(got, *so.attention(host(Q), [host(K)], [host(V)], [0, 150], [150], True, 0.0), "bf16", 150)


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same")])
def test_attention_paged_many_sequences_with_long_ones_among_them(atp, dtype, kind):
    """More sequences than lanes, some of them empty, a few long enough to be cut."""
    rng = np.random.default_rng(55)
    for most_new in (1, 40):
        lengths = rng.integers(0, 40, 150)
        lengths[[3, 90, 149]] = [1500, 700, 1100]
        new = np.minimum(lengths, rng.integers(0, most_new + 1, 150))
        heads, hk, d = 4, 1, 64
        p = Pages(atp, rng, lengths.tolist(), hk, d, 16, dtype, kind)
        Q = randn(rng, (int(new.sum()), heads, d), dtype, 2.0)
        offs = offsets_of(new)
        K, V, present = p.gathered()
        got = host(atp.attention_paged(Q, p.cache, ints(p.table), ints(lengths), ints(offs), max_new=most_new))
        check(got, *so.attention(host(Q), K, V, offs, lengths, True, 0.0, present), dtype, 1500)


def test_thousands_of_sequences(atp):
    rng = np.random.default_rng(56)
    n_seq, heads, hk, d = 5000, 2, 1, 64
    lengths = rng.integers(0, 4, n_seq)
    offs = offsets_of(lengths)
    tokens = int(lengths.sum())
    Q, K, V = (randn(rng, (tokens, h, d), "bf16") for h in (heads, hk, hk))
    k, v = host(K), host(V)
    cut = lambda x: [x[a:a + n] for a, n in so.bounds(offs, tokens)]  # noqa: E731
    want = so.attention(host(Q), cut(k), cut(v), offs, lengths, True, 0.0)
    check(host(atp.attention_packed(Q, K, V, ints(offs))), *want, "bf16", 4)
    p = Pages(atp, rng, lengths.tolist(), hk, d, 1, "bf16", "same", fill=False)
    atp.cache_write(p.cache, K, V, ints(p.table), ints(lengths), ints(offs))
    check(host(atp.attention_paged(Q, p.cache, ints(p.table), ints(lengths), ints(offs))), *want, "bf16", 4)
    back, _ = atp.cache_read(p.cache, ints(p.table), ints(lengths), ints(offs), tokens=tokens)
    assert torch.equal(back, K)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_that_make_no_sense_stay_within_the_tensors(atp, dtype):
    """Decreasing and far offsets: nothing is read or written outside, whatever is computed."""
    rng = np.random.default_rng(57)
    heads, hk, d, tokens = 4, 2, 64, 64
    p = Pages(atp, rng, [700, 64, 64, 64, 64, 64], hk, d, 16, dtype, "same")
    wide = torch.full((tokens + 40, heads, d), 5.0, dtype=TORCH[dtype], device="cuda")
    out = wide[20:20 + tokens]
    Q, K, V = randn(rng, (tokens, heads, d), dtype), randn(rng, (tokens, hk, d), dtype), randn(rng, (tokens, hk, d), dtype)
    for offs in ([0, 64, 0, 64, 0, 64, 0], [-5, 30, 10, 2 ** 31 - 1, -2 ** 31, 64, 64], [64, 0, 64, 0, 64, 0, 64]):
        o = ints(offs)
        args = (ints(p.table), ints([700, 64, 64, 64, 64, 64]), o)
        atp.attention_packed(Q, K, V, o, out=out)
        atp.attention_paged(Q, p.cache, *args, out=out)
        atp.cache_read(p.cache, *args, out=(out[:, :hk], out[:, hk:]))
        spare = sorted(set(range(p.n_pages)) - set(p.table.ravel().tolist()))
        before = p.cache.K[spare].clone()
        atp.cache_write(p.cache, K, V, *args)
        torch.cuda.synchronize()
        assert (wide[:20] == 5.0).all() and (wide[20 + tokens:] == 5.0).all() and torch.isfinite(wide).all()
        assert torch.equal(p.cache.K[spare], before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_the_same_type_are_moved_bit_by_bit(atp, dtype):
    gen = torch.Generator("cuda").manual_seed(58)
    as_int = torch.int16 if dtype == "bf16" else torch.int32
    bits = torch.randint(-2 ** 15 if dtype == "bf16" else -2 ** 31, 2 ** 15 if dtype == "bf16" else 2 ** 31, (90, 6, 64), generator=gen, device="cuda", dtype=torch.int64).to(as_int)
    x = bits.view(TORCH[dtype])
    cache = atp.PagedCache.empty(6, 3, 16, 64, TORCH[dtype])
    args = (ints([[5, 0, 3, 1, 4, 2]]), ints([90]), ints([0, 90]))
    atp.cache_write(cache, x[:, :3], x[:, 3:], *args)
    K, V = atp.cache_read(cache, *args, tokens=90)
    assert torch.equal(K.view(as_int), bits[:, :3]) and torch.equal(V.view(as_int), bits[:, 3:])


def test_values_that_are_not_finite_in_a_long_prompt_cost_no_more_than_their_tile(atp):
    """A spoilt value far behind in a long prompt: the rows before it are as they should be, and the call stays quick."""
    rng = np.random.default_rng(59)
    n, heads, d = 6000, 2, 128
    Q, K, V = (randn(rng, (n, heads, d), "bf16") for _ in range(3))
    offs = ints([0, n])
    clean = atp.attention_packed(Q, K, V, offs)
    V[5500, :, 7] = float("inf")
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    atp.attention_packed(Q, K, V, offs)
    start.record()
    got = atp.attention_packed(Q, K, V, offs)
    end.record()
    torch.cuda.synchronize()
    same = (got[:5400] == clean[:5400]).all() and torch.isfinite(got[:5500]).all() and not torch.isfinite(got[5500:, :, 7]).any()
    assert same
    rest = torch.arange(d, device="cuda") != 7
    assert (got[..., rest].float() - clean[..., rest].float()).abs().max() <= 2 ** -7 * clean.float().abs().max()
    assert start.elapsed_time(end) < 20.0


WIDTHS = [
    # lengths, new tokens, heads, kv_heads, d_h, page size: widths that are no multiple of 16, many heads to a key head, wide tables
    ([300, 20], [1, 1], 128, 1, 72, 32),
    ([300, 20], [150, 3], 4, 2, 104, 64),
    ([150, 90], [40, 90], 2, 1, 200, 16),
    ([260], [7], 96, 2, 24, 128),
    ([1200, 70], [1, 1], 16, 2, 200, 64),
]


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
@pytest.mark.parametrize("case", WIDTHS, ids=str)
def test_attention_of_odd_widths_with_a_scale_of_its_own_into_column_blocks(atp, dtype, kind, case):
    lengths, new, heads, hk, d, page = case
    rng = np.random.default_rng(61)
    p = Pages(atp, rng, lengths, hk, d, page, dtype, kind, most=-(-max(lengths) // page) + 5)
    for s, n in enumerate(lengths):   # what stands behind a sequence's pages is not looked at
        p.table[s, -(-n // page):] = rng.choice([-1, 0, 2 ** 31 - 1, -2 ** 31])
    offs = offsets_of(new)
    Q = randn(rng, (sum(new), heads, d), dtype, 2.0)
    K, V, present = p.gathered()
    wide = torch.full((sum(new), heads + 3, d), 9.0, dtype=TORCH[dtype], device="cuda")
    for scale in (0.02, 1.0):
        got = atp.attention_paged(Q, p.cache, ints(p.table), ints(lengths), ints(offs), scale=scale, out=wide[:, 2:2 + heads])
        check(host(got), *so.attention(host(Q), K, V, offs, lengths, True, scale, present), dtype, max(lengths))
        assert (wide[:, :2] == 9.0).all() and (wide[:, 2 + heads:] == 9.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [24, 72, 104, 200])
def test_attention_packed_of_odd_widths(atp, dtype, d):
    rng = np.random.default_rng(62)
    for lengths, heads, hk in (([150, 7], 6, 2), ([20, 1, 9], 64, 1)):
        tokens, offs = sum(lengths), offsets_of(lengths)
        Q, K, V = (randn(rng, (tokens, h, d), dtype, 1.5) for h in (heads, hk, hk))
        wide = torch.full((tokens, heads + 1, d), 9.0, dtype=TORCH[dtype], device="cuda")
        got = host(atp.attention_packed(Q, K, V, ints(offs), scale=0.1, out=wide[:, 1:]))
        k, v = host(K), host(V)
        cut = lambda x: [x[a:a + n] for a, n in so.bounds(offs, tokens)]  # noqa: E731
        check(got, *so.attention(host(Q), cut(k), cut(v), offs, lengths, True, 0.1), dtype, max(lengths))
        assert (wide[:, 0] == 9.0).all()


def test_two_captured_calls_share_a_workspace(atp):
    """Two graphs over one workspace, replayed in turn with eager work between them, give what eager calls give."""
    rng = np.random.default_rng(63)
    p = Pages(atp, rng, [3000, 500], 2, 64, 64, "bf16", "e4m3")
    table, length, offs = ints(p.table), ints([3000, 500]), ints([0, 1, 2])
    Q = [randn(rng, (2, 8, 64), "bf16") for _ in range(2)]
    ws = torch.empty(atp.attention_paged_workspace(p.cache, 2, table.shape[1], 2, 8, torch.bfloat16, 1), dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(q) for q in Q]
    call = lambda i: atp.attention_paged(Q[i], p.cache, table, length, offs, max_new=1, workspace=ws, out=out[i])  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(0)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(i)
    for _ in range(3):
        for i in range(2):
            Q[i].copy_(randn(rng, Q[i].shape, "bf16"))
            ws.fill_(255)   # what the workspace held does not matter
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(out[i], atp.attention_paged(Q[i], p.cache, table, length, offs, max_new=1))


@pytest.mark.parametrize("dtype,kind", [("bf16", "same"), ("bf16", "e4m3"), ("f32", "same"), ("f32", "e4m3")])
@pytest.mark.parametrize("what", ["K", "V"])
def test_values_that_are_nan_reach_the_sum_from_a_part_of_the_keys_that_weighs_nothing(atp, dtype, kind, what):
    """Key 4000 outweighs every other by more than the exponents of 32 bits; a NaN at key 100, in another share of the keys, still makes NaN: of
    every feature when it stands in the key, of its own feature in the value."""
    rng = np.random.default_rng(31)
    n, heads, d, page = 4096, 2, 64, 64
    K, V, Q = randn(rng, (n, 1, d), dtype), randn(rng, (n, 1, d), dtype), randn(rng, (1, heads, d), dtype)
    Q[:, :, 0], K[:, :, 0], K[4000, :, 0] = 40.0, 0.0, 400.0
    (K if what == "K" else V)[100, 0, 5] = float("nan")
    cache = atp.PagedCache.empty(n // page, 1, page, d, torch.float8_e4m3fn if kind == "e4m3" else TORCH[dtype])
    table = ints(np.arange(n // page)[None])
    atp.cache_write(cache, K, V, table, ints([n]), ints([0, n]))
    print(f"nan {dtype} {kind} {what}", flush=True)
    got = host(atp.attention_paged(Q, cache, table, ints([n]), ints([0, 1])))
    nan = np.ones(d, bool) if what == "K" else np.arange(d) == 5
    assert np.array_equal(np.isnan(got), np.broadcast_to(nan, got.shape))
    code = host(V[4000, 0]) if kind == "same" else host(atp.cache_read(cache, table, ints([4001]), ints([0, 1]), tokens=1, dtype=torch.float32)[1][0, 0])
    if what == "V":
        assert np.abs(got - code)[..., ~nan].max() <= HALF[dtype] * 4 * np.abs(code).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_workgroups_than_a_row_of_the_grid_holds(atp, dtype):
    """512 sequences of one token, 32768 heads: more than 2^24 workgroups.  A single key weighs 1, so every head gives its value."""
    n, heads, d = 512, 32768, 8
    gen = torch.Generator(device="cuda").manual_seed(5)
    Q, K, V = (torch.randn((n, heads, d), dtype=TORCH[dtype], device="cuda", generator=gen) for _ in range(3))
    print(f"workgroups {dtype}", flush=True)
    assert torch.equal(atp.attention_packed(Q, K, V, ints(np.arange(n + 1))), V)


def test_more_tokens_than_a_row_of_the_grid_holds(atp):
    """2^26 + 1000 tokens of one head: written and read bit by bit."""
    n, page = 2 ** 26 + 1000, 65536
    pages = (n + page - 1) // page
    print("tokens", flush=True)
    bits = torch.arange(n * 4, dtype=torch.int32, device="cuda")
    K, V = bits.view(torch.bfloat16).view(n, 1, 8), (bits ^ 0x55555555).view(torch.bfloat16).view(n, 1, 8)
    cache = atp.PagedCache.empty(pages, 1, page, 8, torch.bfloat16)
    table = ints(np.random.default_rng(6).permutation(pages)[None])
    out = torch.zeros_like(K), torch.zeros_like(V)
    atp.cache_write(cache, K, V, table, ints([n]), ints([0, n]))
    atp.cache_read(cache, table, ints([n]), ints([0, n]), out=out)
    as_bits = lambda t: t.view(-1).view(torch.int32)  # noqa: E731
    assert torch.equal(as_bits(out[0]), as_bits(K)) and torch.equal(as_bits(out[1]), as_bits(V))


# ------------------------------------------------------------------ refusals of the binding
def test_refusals(atp):
    bf = torch.bfloat16
    e = lambda *s, dtype=bf: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    offs, length, table = ints([0, 4]), ints([4]), ints([[0]])
    cache = atp.PagedCache.empty(1, 2, 16, 64, bf)
    with pytest.raises(ValueError):
        atp.attention_packed(e(4, 4, 64).cpu(), e(4, 2, 64), e(4, 2, 64), offs)
    with pytest.raises(ValueError):
        atp.attention_packed(e(4, 4, 64), e(4, 2, 64), e(5, 2, 64), offs)
    with pytest.raises(ValueError):
        atp.attention_packed(e(4, 4, 64), e(4, 2, 64), e(4, 2, 64), offs.long())
    with pytest.raises(ValueError):
        atp.attention_packed(e(4, 4, 128)[..., ::2], e(4, 2, 64), e(4, 2, 64), offs)
    with pytest.raises(ValueError):
        atp.attention_packed(e(4, 4, 64), e(4, 2, 64, dtype=torch.float32), e(4, 2, 64), offs)
    with pytest.raises(atp.AtpError):
        atp.attention_packed(e(4, 3, 64), e(4, 2, 64), e(4, 2, 64), offs)       # 3 heads over 2
    with pytest.raises(atp.AtpError):
        atp.attention_packed(e(4, 4, 68), e(4, 2, 68), e(4, 2, 68), offs)       # rows of no multiple of 16 bytes, width no multiple of 8
    with pytest.raises(atp.AtpError):
        atp.attention_packed(e(4, 2, 264), e(4, 2, 264), e(4, 2, 264), offs)    # too wide
    with pytest.raises(ValueError):
        atp.PagedCache(e(1, 2, 16, 64).to(torch.float8_e4m3fn), e(1, 2, 16, 64).to(torch.float8_e4m3fn))
    with pytest.raises(ValueError):
        atp.PagedCache(e(1, 2, 16, 64), e(1, 2, 16, 32))
    with pytest.raises(atp.AtpError):
        atp.cache_write(atp.PagedCache.empty(1, 2, 24, 64, bf), e(4, 2, 64), e(4, 2, 64), table, length, offs)   # page size
    with pytest.raises(ValueError):
        atp.cache_write(cache, e(4, 2, 64, dtype=torch.float32), e(4, 2, 64, dtype=torch.float32), table, length, offs)
    with pytest.raises(ValueError):
        atp.cache_read(cache, table, length, offs)
    with pytest.raises(ValueError):
        atp.attention_paged(e(4, 4, 64), cache, table, ints([4, 4]), offs)
    assert atp.attention_packed(e(0, 4, 64), e(0, 2, 64), e(0, 2, 64), ints([0, 0])).shape == (0, 4, 64)
    atp.cache_write(cache, e(0, 2, 64), e(0, 2, 64), table, length, ints([0, 0]))
