"""Chunk attention at the ends of its range: logits and values that are finite but very large, keys that a row does not see with any
contents, keys that are left out."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import chunk_harness as C

BITS = pytest.mark.parametrize("bits", [16, 8])


def _steps(n, H_kv, top, seed=0):
    """n keys (bf16-exact, n <= 900) that are multiples b = 1 .. of one pattern of signs, in random order, the largest and the smallest
    twice; with queries that are multiples of the pattern the products are whole numbers times a power of two, exact in single precision,
    and any two that differ do so by 2^-8 or more of themselves.  -> keys [n, H_kv, 128], the pattern, a factor: queries of up to 15
    times it times the pattern have logits of up to 2^top."""
    g = torch.Generator().manual_seed(seed)
    sign = (torch.randint(0, 2, (128,), generator=g) * 2 - 1).float()
    b = 1 + torch.randint(0, 127, (n,), generator=g).float()
    order = torch.randperm(n, generator=g)
    b[order[0]] = b[order[1 % n]] = 128.0
    if n > 4:
        b[order[2]] = b[order[3]] = 0.5
    half = top // 2
    k = (b[:, None] * sign * 2.0 ** (half - 12))[:, None].expand(n, H_kv, 128).contiguous()
    return k, sign, 2.0 ** (top - half - 2)


def _check(cache, q, m, mask, out, lse):
    """By the definition: distinct logits are so far apart that a row is the mean over its largest, whose products are equal bit by bit.
    Output as in chunk_harness; lse to the fp32 roundings of the logits, 2^-22 of their size (two factors and their product)."""
    ref, mag, rl = C.attend(cache, 0, q, mask)
    got = out.double()
    assert torch.isfinite(got).all()
    assert ((got - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS).all(), float((got - ref).abs().max())
    assert ((lse.double() - rl).abs() <= C.LSE_ABS + rl.abs() * 2.0 ** -21).all()


TOPS = pytest.mark.parametrize("top", [16, 20, 24, 26, 27, 28, 29, 30, 31, 32, 34, 40, 64, 100])


def _exact_logits(bits, m, top):
    for n in (m + 3, 700):
        cache = C.Cache([n], 8, 2, 64, bits)
        k, sign, f = _steps(n, 2, top, seed=n + top)
        g = torch.Generator().manual_seed(top)
        cache.put(0, torch.arange(n), k, torch.randn(n, 2, 128, generator=g))
        mult = (torch.randint(1, 16, (m, 8, 1), generator=g) * (torch.randint(0, 2, (m, 8, 1), generator=g) * 2 - 1)).float() * f
        q = (mult * sign).to(torch.bfloat16).cuda()
        for mask in (0, 1):
            out, lse = C.run_attn(cache, q, [m], mask)
            _check(cache, q, m, mask, out, lse)


SIGMAS = pytest.mark.parametrize("sigma", [2.0 ** 11, 1e4, 2e4, 3e4, 1e5, 2.0 ** 30])


def _random_logits(bits, m, sigma):
    """Random queries and keys, sigma times unit normal.  A row whose two largest logits are closer than the products' errors (2^-15 of the
    sum of magnitudes: 128 fp32 additions, each off by less than a step, and over the 8-bit cache the few elements of a query below 2^-10
    of its largest, each off by 2^-17 of that) has no one answer and is only asked to be finite."""
    n = 500
    cache = C.Cache([n], 8, 2, 64, bits)
    g = torch.Generator().manual_seed(int(sigma))
    cache.put(0, torch.arange(n), torch.randn(n, 2, 128, generator=g) * sigma, torch.randn(n, 2, 128, generator=g))
    q = C.queries(m, 8, spread=sigma)
    out, lse = C.run_attn(cache, q, [m], 0)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    ref, mag, rl = C.attend(cache, 0, q, 0)
    k, _ = cache.rows(0)
    x = torch.einsum("mhgd,hnd->mhgn", q.double().view(m, 2, 4, 128), k).reshape(m, 8, n)
    size = torch.einsum("mhgd,hnd->mhgn", q.double().abs().view(m, 2, 4, 128), k.abs()).reshape(m, 8, n).amax(-1)
    two = x.topk(2, -1).values
    clear = two[..., 0] - two[..., 1] > 2.0 ** -14 * size + 2000.0
    assert clear.double().mean() > 0.5
    assert ((out.double() - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS)[clear].all()
    assert ((lse.double() - rl).abs() <= C.LSE_ABS + 2.0 ** -15 * size * 128 ** -0.5).all()


@BITS
@pytest.mark.parametrize("m", [40, 200])
@TOPS
def test_prompt_logits_of_any_finite_size(bits, m, top):
    """Logits up to 2^100 of both signs, rising and falling along the cache, in one tile and over many, split runs and whole ones."""
    _exact_logits(bits, m, top)


@BITS
@SIGMAS
def test_prompt_tokens_of_any_finite_size(bits, sigma):
    _random_logits(bits, 60, sigma)


@BITS
@pytest.mark.parametrize("m", [1, 2, 4])
@TOPS
def test_step_logits_of_any_finite_size(bits, m, top):
    """The same for tiles of eight and sixteen rows."""
    _exact_logits(bits, m, top)


@BITS
@pytest.mark.parametrize("m", [1, 3])
@SIGMAS
def test_step_tokens_of_any_finite_size(bits, m, sigma):
    _random_logits(bits, m, sigma)


@pytest.mark.parametrize("H_q,H_kv,new,row", [(8, 2, 150, 100), (8, 2, 150, 149), (160, 1, 3, 2), (160, 1, 3, 1)])
@pytest.mark.parametrize("big", [2.0 ** 24, 2.0 ** 40, 2.0 ** 90, float("nan")])
@pytest.mark.parametrize("ctx", [0, 333])
def test_values_that_no_query_of_a_tile_sees_change_no_bit(H_q, H_kv, new, row, big, ctx):
    """8-bit cache: the value row of a later token, far larger than all others.  Tiles of queries that lie in front of it (64 tokens with
    four heads a group; one token with 160) give the same bits as with an ordinary row there."""
    n, tile = ctx + new, 64 if H_q == 8 else 1
    cache = C.filled([n], H_q, H_kv, 64, 8)
    q = C.queries(new, H_q)
    want, wl = C.run_attn(cache, q, [new], 1)
    C.check_attn(cache, q, [new], 1, want, wl)
    g = torch.Generator().manual_seed(1)
    cache.put(0, torch.tensor([ctx + row]), torch.randn(1, H_kv, 128, generator=g), torch.randn(1, H_kv, 128, generator=g) * big)
    out, lse = C.run_attn(cache, q, [new], 1)
    before = row // tile * tile
    assert before > 0
    assert torch.equal(out[:before], want[:before]) and torch.equal(lse[:before], wl[:before])
    C.check_attn(cache, q[row:], [new - row], 1, out[row:], lse[row:])


def _check_small(cache, q, m, mask, out, lse):
    """chunk_harness's tolerance without its absolute part, since the values may be as small as they like."""
    ref, mag, rl = C.attend(cache, 0, q, mask)
    assert ((out.double() - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag).all(), float(((out.double() - ref).abs() / mag).max())
    assert ((lse.double() - rl).abs() <= C.LSE_ABS).all()


@pytest.mark.parametrize("new,ctx", [(2, 0), (4, 200), (3, 700), (30, 0), (60, 100), (150, 0), (200, 300)])
@pytest.mark.parametrize("big", [2.0 ** 18, 2.0 ** 22, 2.0 ** 30, 2.0 ** 50, 2.0 ** 90])
@pytest.mark.parametrize("mask", [1, 7])
def test_a_later_token_with_a_far_larger_value_row(new, ctx, big, mask):
    """8-bit cache: rows in front of it, in the same tile of queries, keep their values; rows that see it are about it."""
    n = ctx + new
    cache = C.filled([n], 8, 2, 64, 8)
    g = torch.Generator().manual_seed(new)
    for row in (new - 1, new // 2):
        cache.put(0, torch.tensor([ctx + row]), torch.randn(1, 2, 128, generator=g), torch.randn(1, 2, 128, generator=g) * (big if row == new // 2 else big * big ** 0.1))
    q = C.queries(new, 8)
    out, lse = C.run_attn(cache, q, [new], mask)
    _check_small(cache, q, new, mask, out, lse)


@pytest.mark.parametrize("new,ctx", [(1, 3), (1, 900), (4, 2000), (20, 2), (20, 300), (70, 700), (300, 0)])
@pytest.mark.parametrize("small", [2.0 ** -12, 2.0 ** -24, 2.0 ** -40, 2.0 ** -80])
@pytest.mark.parametrize("where", ["first", "every ninth", "last tile"])
def test_rows_of_zeros_beside_small_values(new, ctx, small, where):
    """8-bit cache: a row of zeros has scale 1, whatever the others have."""
    n = ctx + new
    cache = C.filled([n], 8, 2, 64, 8)
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn(n, 2, 128, generator=g), torch.randn(n, 2, 128, generator=g) * small
    v[{"first": slice(0, 1), "every ninth": slice(None, None, 9), "last tile": slice(n // 128 * 128 + 1, None, 5)}[where]] = 0.0
    cache.put(0, torch.arange(n), k, v)
    q = C.queries(new, 8)
    for mask in (0, 1):
        out, lse = C.run_attn(cache, q, [new], mask)
        _check_small(cache, q, new, mask, out, lse)


@pytest.mark.parametrize("new,ctx", [([3], [400]), ([50], [400]), ([50, 2, 130], [400, 3000, 0])])
def test_scales_of_very_different_size_with_large_logits(new, ctx):
    """8-bit cache: the reference of the exponentials and that of the scales move in the same tiles."""
    lens = [c + m for c, m in zip(ctx, new)]
    cache = C.filled(lens, 8, 2, 16, 8)
    g = torch.Generator().manual_seed(5)
    for p, n in enumerate(lens):
        size = torch.exp2(torch.randint(-45, 46, (n, 1, 1), generator=g).float())
        cache.put(p, torch.arange(n), 20 * torch.randn(n, 2, 128, generator=g), size * torch.randn(n, 2, 128, generator=g))
    q = C.queries(sum(new), 8)
    out, lse = C.run_attn(cache, q, new, 1)
    s = C.starts(new)
    for p, m in enumerate(new):
        ref, mag, rl = C.attend(cache, p, q[s[p]:s[p + 1]], 1)
        d = 20 * C.LSE_ABS                                   # logits twenty times as large
        assert ((out[s[p]:s[p + 1]].double() - ref).abs() <= C.OUT_REL * ref.abs() + (C.W_REL + 2 * d) * mag).all()
        assert ((lse[s[p]:s[p + 1]].double() - rl).abs() <= d).all()


@pytest.mark.parametrize("new,ctx,row", [(2, 0, 1), (4, 50, 2), (40, 0, 30), (40, 90, 39), (150, 300, 140)])
@pytest.mark.parametrize("scale", [float("inf"), 3.0e38, 2.0 ** 121, float("nan")])
def test_a_value_scale_that_is_none_behind_the_mask(new, ctx, row, scale):
    """8-bit cache: rows that do not see the key are as with an ordinary scale."""
    cache = C.filled([ctx + new], 8, 2, 64, 8)
    q = C.queries(new, 8)
    want, wl = C.run_attn(cache, q, [new], 1)
    page = cache.table[0, (ctx + row) // 64]
    cache.vs[page, :, (ctx + row) % 64] = scale
    out, lse = C.run_attn(cache, q, [new], 1)
    assert torch.equal(out[:row], want[:row]) and torch.equal(lse, wl)


@BITS
@pytest.mark.parametrize("m", [1, 30, 150])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 40, 2.0 ** 70])
@pytest.mark.parametrize("rise", [20, 60, 120])
def test_large_values_under_a_steep_rise(bits, m, size, rise):
    """Logits that rise by up to 2^rise along a tile and from tile to tile, values of any size: the sum of P v stays finite."""
    n = m + 400
    cache = C.Cache([n], 8, 2, 64, bits)
    g = torch.Generator().manual_seed(rise)
    step = torch.arange(n).float()
    for at in (0, 128, 300):                                 # the first half of a tile flat, then up, down again behind
        step[at:at + 96] = -1.0
    up = torch.where(step < 0, torch.zeros(n), (step % 128) / 128 * rise * 0.6931 / (128 * 0.25 * 128 ** -0.5))
    k = (0.25 + torch.randn(n, 2, 128, generator=g) * 0.01) * up[:, None, None]
    cache.put(0, torch.arange(n), k, torch.randn(n, 2, 128, generator=g) * size)
    q = (1.0 + 0.01 * torch.randn(m, 8, 128, generator=g)).to(torch.bfloat16).cuda()
    for mask in (0, 1):
        out, lse = C.run_attn(cache, q, [m], mask)
        ref, mag, rl = C.attend(cache, 0, q, mask)
        d = rise * 2.0 ** -14                                # fp32 additions of 128 products of one sign, the 8-bit query's codes, the factors
        assert ((out.double() - ref).abs() <= C.OUT_REL * ref.abs() + (C.W_REL + 2 * d) * mag).all()
        assert ((lse.double() - rl).abs() <= d).all()


@BITS
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("new", [[1, 1], [4, 2], [40, 1], [300, 70], [2, 200]])
@pytest.mark.parametrize("n", [300, 9000])
def test_rows_whose_every_key_is_left_out(bits, page, new, n):
    """Problem 0 has no valid page at all, problem 1 none in its first 256 positions: rows without a key are 0 with lse -inf, the others
    as if the keys were not there; whole results and ones merged from few and many parts."""
    import paper_2602_14209_b200.binding as mb
    lens = [n, 320]
    cache = C.filled(lens, 8, 2, page, bits)
    q = C.queries(sum(new), 8)
    table = cache.table.clone()
    cache.table[0] = -1
    cache.table[1, :256 // page] = 10 ** 6
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = C.run_attn(cache, q, new, 1, status=status)
    assert int(status.item()) == mb.DEV_BAD_PAGE
    m0 = new[0]
    assert (out[:m0] == 0).all() and (lse[:m0] == float("-inf")).all()
    dead = max(0, 256 - (320 - new[1]))                      # rows of problem 1 in front of position 256
    assert (out[m0:m0 + dead] == 0).all() and (lse[m0:m0 + dead] == float("-inf")).all()
    cache.table.copy_(table)
    k, v = (x[:, 256:] for x in cache.rows(1))
    for i in range(dead, new[1]):
        e = 320 - new[1] + i + 1 - 256
        x = torch.einsum("hgd,hnd->hgn", q[m0 + i].double().view(2, 4, 128), k[:, :e]) * 128 ** -0.5
        w = torch.softmax(x, -1)
        ref, mag = (torch.einsum("hgn,hnd->hgd", w, y).reshape(8, 128) for y in (v[:, :e], v[:, :e].abs()))
        assert ((out[m0 + i].double() - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS).all()
        assert ((lse[m0 + i].double() - torch.logsumexp(x, -1).reshape(8)).abs() <= C.LSE_ABS).all()


@BITS
def test_a_bound_of_no_new_tokens(bits):
    """max_len 0: empty ranges are as it says, others are reported like any that exceed the bound; nothing is written."""
    import paper_2602_14209_b200.binding as mb
    cache = C.filled([70, 90], 8, 2, 64, bits)
    x = C.queries(6, 8)
    pools = [t.clone() for t in ((cache.k, cache.v) if bits == 16 else (cache.k, cache.v, cache.ks, cache.vs))]
    attn, append = (mb.mage_chunk_attn, mb.mage_append_chunk) if bits == 16 else (mb.mage_chunk_attn_kv8, mb.mage_append_chunk_kv8)
    for starts, want in (([0, 0, 0], 0), ([0, 0, 5], mb.DEV_BAD_CHUNK)):
        chunk = mb.ChunkBatch(cache.kv, torch.tensor(starts, dtype=torch.int32, device="cuda"), 6, max_len=0)
        out, status = torch.full((6, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        attn(cache.kv, chunk, x, 128 ** -0.5, out, chunk.new_workspace(), dev_status=status)
        assert int(status.item()) == want and (out == 7.0).all()
        status.zero_()
        append(cache.kv, chunk, x[:, :2], x[:, 2:4], dev_status=status)
        assert int(status.item()) == want
    for a, b in zip(pools, (cache.k, cache.v) if bits == 16 else (cache.k, cache.v, cache.ks, cache.vs)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_rows_read_back_are_rounded_twice():
    """bf16 of the single-precision product: of 2^23 random scales and codes, those where one rounding of the exact product differs."""
    import paper_2602_14209_b200.binding as mb
    g = torch.Generator().manual_seed(0)
    s = torch.randint(2 ** 23, 2 ** 24, (2 ** 16,), generator=g).float() * 2.0 ** -24     # (whole numbers: the same on every machine)
    code = torch.randint(0, 127, (2 ** 16, 128), generator=g).to(torch.uint8)
    x = code.view(torch.float8_e4m3fn).double() * s.double()[:, None]        # exact: 4 + 24 bits
    twice = x.float().to(torch.bfloat16)
    m, e = torch.frexp(x)
    once = torch.ldexp(torch.round(m * 256), e - 8)                                      # (to nearest, ties to even, in 64 bits)
    odd = once != twice.double()
    assert int(odd.sum()) >= 8                                               # there are such elements
    odd = odd.any(1)
    n = int(odd.sum())
    cache = C.Cache([n], 1, 1, 0, 8)
    for pool, sc in ((cache.k, cache.ks), (cache.v, cache.vs)):
        pool[0, 0], sc[0, 0] = code[odd].cuda(), s[odd].cuda()
    ko, vo = (torch.empty(1, 1, n, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv8_read(cache.kv, ko, vo)
    assert torch.equal(ko[0, 0].cpu(), twice[odd]) and torch.equal(vo[0, 0].cpu(), twice[odd])


@pytest.mark.parametrize("new,ctx", [([1], [0]), ([1, 1], [20, 9000]), ([4, 2], [0, 300]), ([40], [0]), ([150, 30], [0, 2000]), ([300], [900])])
@pytest.mark.parametrize("which", ["all", "first", "every third", "last"])
@pytest.mark.parametrize("value", [1.0, float("inf")])
def test_logits_of_minus_infinity(new, ctx, which, value):
    """16-bit cache: keys that are not left out but have logits of -inf.  Beside others they have weight 0 (and 0 * inf is NaN, in the columns
    of an infinite value); a row that sees no others is 0 / 0, unlike one whose keys are left out, with lse -inf either way."""
    lens = [c + m for c, m in zip(ctx, new)]
    cache = C.filled(lens, 8, 2, 64, 16)
    g = torch.Generator().manual_seed(7)
    for p, n in enumerate(lens):
        j = {"all": torch.arange(n), "first": torch.arange(min(n, 140)), "every third": torch.arange(0, n, 3), "last": torch.arange(n - 1, n)}[which]
        k, v = torch.randn(len(j), 2, 128, generator=g), torch.randn(len(j), 2, 128, generator=g)
        k[..., 5] = float("-inf")
        v[..., 9] *= value
        cache.put(p, j, k, v)
    q = C.queries(sum(new), 8)
    q[..., 5] = 1.0
    out, lse = C.run_attn(cache, q, new, 1)
    C.check_attn(cache, q, new, 1, out, lse)
