"""The 4-bit cache: rows written, read back and attended, against its definition in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import chunk_harness as C
import kv4_harness as K4
from paper_2602_14209_b200 import binding as mb


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def _append(cache, new, k, v, status=None, max_len=None):
    chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), k.shape[0], max_len=max(new) if max_len is None else max_len)
    mb.mage_append_chunk_kv4(cache.kv, chunk, k, v, dev_status=status)


def _pools(c):
    return [x.clone() for x in (c.k, c.v, c.ks, c.vs)]


def _rows_to_write(n, H_kv, seed):
    """Rows as a model makes them, and rows where the rounding decides: zeros, halves, huge and tiny ones, powers of two of all sizes."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, H_kv, 128, generator=g)
    kind = torch.randint(0, 8, (n, H_kv, 8), generator=g).repeat_interleave(16, -1)
    size = 2.0 ** torch.randint(-30, 18, (n, H_kv, 8), generator=g).repeat_interleave(16, -1).float()
    whole = torch.randint(-255, 256, (n, H_kv, 128), generator=g).float()
    x = torch.where(kind == 1, torch.zeros(()), x)
    x = torch.where(kind == 2, x * size, x)
    x = torch.where(kind == 3, whole * size / 64, x)                      # many halves among them
    x = torch.where(kind == 4, x * 1e30, x)
    x = torch.where(kind == 5, x * 1e-36, x)
    x = torch.where(kind == 6, torch.round(x * 4) / 2 * size, x)
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("page,token_major", [(0, False), (0, True), (16, False), (64, False)])
@pytest.mark.parametrize("H_kv", [1, 3, 8])
@pytest.mark.parametrize("new", [[1], [5, 0, 1, 33], [700, 1, 0, 550]])
def test_append_by_the_definition(page, token_major, H_kv, new):
    ctx = [7, 0, 64, 31][:len(new)]
    cache = K4.Cache([c + m for c, m in zip(ctx, new)], H_kv * 2, H_kv, page, n_max=760, seed=H_kv, token_major=token_major)
    n, s = sum(new), C.starts(new)
    x = torch.zeros(n + 2, 2 * H_kv + 1, 128, dtype=torch.bfloat16)
    x[:n, :H_kv], x[:n, H_kv:2 * H_kv] = _rows_to_write(n, H_kv, 1), _rows_to_write(n, H_kv, 2)
    if n > 5:
        x[2, 0, 77], x[3, H_kv, 5], x[4, 0, 127] = float("nan"), float("inf"), float("-inf")
    x = x.cuda()
    before, status = _pools(cache), _status()
    _append(cache, new, x[:, :H_kv], x[:, H_kv:2 * H_kv], status, max_len=max(new))
    assert int(status.item()) == 0
    want = before
    for p, m in enumerate(new):
        if m == 0:
            continue
        i = cache.at(p, torch.arange(ctx[p], ctx[p] + m))
        for which, first in ((0, 0), (1, H_kv)):
            c, u = K4.quantise(x[s[p]:s[p + 1], first:first + H_kv])
            c = K4.pack(c).cuda()
            u = u.cuda()
            if not page:
                c, u = c.transpose(0, 1), u.transpose(0, 1)
            want[which][i], want[2 + which][i] = c, u
    for got, ref in zip(_pools(cache), want):
        assert torch.equal(got, ref)


def test_append_every_bf16_number():
    """Each finite bf16 number as the largest of a group, with halves and quarters of it and their neighbours beside it."""
    bits = torch.arange(0, 0x7F80, dtype=torch.int32)
    top = bits.to(torch.int16).view(torch.bfloat16)
    pad = -(-top.numel() // 8) * 8
    top = torch.cat([top, top[:pad - top.numel()]])
    frac = torch.tensor([1, 13 / 14, 11 / 14, 9 / 14, 0.5, 5 / 14, 3 / 14, 1 / 14, 15 / 16, 7 / 8, 3 / 4, 1 / 4, 1 / 8, 0.07, 0.072, 0.65])
    x = (top.float()[:, None] * frac * torch.tensor([1.0, -1.0] * 8)).to(torch.bfloat16).reshape(-1, 1, 128)
    n = x.shape[0]
    cache = K4.Cache([n], 1, 1, 0)
    _append(cache, [n], x.cuda(), (-x).cuda())
    for y, pool, sc in ((x, cache.k, cache.ks), (-x, cache.v, cache.vs)):
        c, u = K4.quantise(y)
        assert torch.equal(pool[0, 0].cpu(), K4.pack(c)[:, 0]) and torch.equal(sc[0, 0].cpu(), u[:, 0])


def test_append_refuses_what_has_no_place():
    cache = K4.filled([40, 20, 9], 4, 2, 16, n_max=48)
    cache.seq_lens.copy_(torch.tensor([49, 20, 3]))                  # too long, fine, shorter than its new tokens
    cache.table[1, 1] = 99
    before, status = _pools(cache), _status()
    x = torch.randn(14, 2, 128, device="cuda").to(torch.bfloat16)
    _append(cache, [4, 6, 4], x, x, status)
    assert int(status.item()) == mb.DEV_CACHE_FULL | mb.DEV_BAD_PAGE
    i = cache.at(1, torch.arange(14, 16))                            # rows 14 .. 19: the last four are on the bad page
    c, u = K4.quantise(x[4:6])
    for pool, old, new in zip(_pools(cache), before, (K4.pack(c), K4.pack(c), u, u)):
        old[i] = new.cuda()
        assert torch.equal(pool, old)
    status.zero_()
    chunk = mb.ChunkBatch(cache.kv, torch.tensor([0, 9, 4, 99], dtype=torch.int32, device="cuda"), 14, max_len=6)
    mb.mage_append_chunk_kv4(cache.kv, chunk, x, x, dev_status=status)
    assert int(status.item()) & mb.DEV_BAD_CHUNK
    for pool, old in zip(_pools(cache), before):
        assert torch.equal(pool, old)


@pytest.mark.parametrize("page", [0, 16, 64])
def test_read(page):
    lens, H_kv = [70, 0, 1, 333], 3
    cache = K4.filled(lens, 6, H_kv, page, seed=4, n_max=400)
    i = cache.at(3, torch.tensor([17]))
    cache.ks[i] = 255
    for begin, rows in ((0, 400), (5, 77), (332, 1), (399, 2)):
        k, v = (torch.full((4, H_kv, rows, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        mb.mage_kv4_read(cache.kv, k, v, row_begin=begin)
        for p, n in enumerate(lens):
            m = max(0, min(rows, n - begin))
            rk, rv = cache.rows(p)
            torch.testing.assert_close(k[p, :, :m].double(), rk[:, begin:begin + m], rtol=0, atol=0, equal_nan=True)
            assert torch.equal(v[p, :, :m].double(), rv[:, begin:begin + m])
            assert (k[p, :, m:] == 7.0).all() and (v[p, :, m:] == 7.0).all()
    pick = torch.full((4, H_kv, 9), -1, dtype=torch.int32, device="cuda")
    pick[0], pick[3] = torch.tensor([3, 3, 69, 0, 5, 6, 7, 8, 70]), torch.tensor([332, 0, 16, 18, 1, 2, 3, 4, -5])
    pick[2, :, 0] = 0
    k_eff, status = torch.tensor([9, 0, 1, 9], dtype=torch.int32, device="cuda"), _status()
    k, v = (torch.full((4, H_kv, 9, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv4_read(cache.kv, k, v, indices=pick, k_eff=k_eff, dev_status=status)
    assert int(status.item()) == mb.DEV_BAD_INDEX
    for p, m in ((0, 8), (1, 0), (2, 1), (3, 8)):
        rk, rv = cache.rows(p)
        for h in range(H_kv):
            assert torch.equal(k[p, h, :m].double(), rk[h][pick[p, h, :m].long()]) and torch.equal(v[p, h, :m].double(), rv[h][pick[p, h, :m].long()])
        assert (k[p, :, m:] == 7.0).all() and (v[p, :, m:] == 7.0).all()


def test_every_code_under_every_scale():
    """All sixteen codes (the unused one, too) under all scale bytes, read back and as values of an attention that sees one key."""
    u = torch.arange(256, dtype=torch.uint8).reshape(-1, 1).expand(256, 8).contiguous().cuda()
    codes = torch.stack([K4.pack((torch.arange(128) + r) % 16 - 8) for r in range(256)]).cuda()
    cache = K4.Cache([1] * 256, 1, 1, 0)
    for pool, sc in ((cache.k, cache.ks), (cache.v, cache.vs)):
        pool[:, 0, 0], sc[:, 0, 0] = codes, u
    k, v = (torch.zeros(256, 1, 1, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv4_read(cache.kv, k, v)
    want = K4.values(codes, u)
    for got in (k, v):
        torch.testing.assert_close(got[:, 0, 0].double(), want, rtol=0, atol=0, equal_nan=True)
    assert torch.isnan(k[248:].float()).all() and torch.isfinite(k[:248].float()).all()
    cache.ks[:] = 100                                                    # (keys that are numbers)
    for heads in (1, 40):                                                # by both kernels
        wide = mb.Kv4Cache(cache.k, cache.v, cache.ks, cache.vs, heads, seq_lens=cache.seq_lens)
        q = torch.randn(256, heads, 128, device="cuda").to(torch.bfloat16)
        chunk = mb.ChunkBatch(wide, torch.arange(257, dtype=torch.int32, device="cuda"), 256, max_len=1)
        out = torch.empty_like(q)
        mb.mage_chunk_attn_kv4(wide, chunk, q, 0.1, out, chunk.new_workspace())
        torch.testing.assert_close(out.double(), want[:, None].expand(-1, heads, -1), rtol=0, atol=0, equal_nan=True)


HEADS = [(8, 2), (28, 4), (5, 1), (3, 3), (16, 1)]


@pytest.mark.parametrize("mask", [0, 1, 7, 32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("lens,new", [([1, 2, 40], [1, 1, 1]), ([129, 31, 0, 700], [1, 2, 0, 1]), ([1000, 6, 257], [3, 3, 2])])
def test_attention_of_few_rows(mask, heads, page, lens, new):
    cache = K4.filled(lens, *heads, page, seed=len(lens), n_max=max(lens) + 9)
    q = C.queries(sum(new), heads[0])
    out, lse = K4.run_attn(cache, q, new, mask)
    C.check_attn(cache, q, new, mask, out, lse)


@pytest.mark.parametrize("mask", [0, 1, 32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [0, 16, 128])
@pytest.mark.parametrize("lens,new", [([300], [300]), ([129, 31, 0, 700], [129, 20, 0, 333]), ([2000, 64, 1], [70, 64, 1])])
def test_attention_of_chunks(mask, heads, page, lens, new):
    cache = K4.filled(lens, *heads, page, seed=len(lens) + 7, n_max=max(lens) + 5)
    q = C.queries(sum(new) + 3, heads[0])
    out, lse = K4.run_attn(cache, q, new, mask)
    C.check_attn(cache, q, new, mask, out, lse)


@pytest.mark.parametrize("lens,new,heads", [([20000], [1], (8, 2)), ([30000, 100, 1], [2, 1, 1], (28, 4)), ([20011], [40], (28, 4)), ([9000, 4000], [300, 100], (8, 1))])
def test_attention_over_long_caches(lens, new, heads):
    """Items cut over many runs."""
    cache = K4.filled(lens, *heads, 64, seed=5)
    q = C.queries(sum(new), heads[0], spread=2.0)
    out, lse = K4.run_attn(cache, q, new, 1)
    C.check_attn(cache, q, new, 1, out, lse)
    again, _ = K4.run_attn(cache, q, new, 1)
    assert torch.equal(out, again)


def test_attention_of_a_token_major_cache():
    cache = K4.filled([300, 77], 8, 2, 0, token_major=True)
    for new in ([1, 1], [100, 50]):
        q = C.queries(sum(new), 8)
        out, lse = K4.run_attn(cache, q, new, 1)
        C.check_attn(cache, q, new, 1, out, lse)


@pytest.mark.parametrize("new", [[2, 3], [120, 40]])
@pytest.mark.parametrize("mask", [1, 32, 0])
def test_rows_of_nan(new, mask):
    """Keys and values that hold no number: NaN for the rows that see them, no trace in the others."""
    cache = K4.filled([200, 90], 8, 2, 16, seed=11)
    for p, j, what in ((0, 197, "v"), (0, 199, "k"), (1, 60, "v"), (1, 89, "k")):
        i = cache.at(p, torch.tensor([j]))
        (cache.vs if what == "v" else cache.ks)[i] = 255
        (cache.v if what == "v" else cache.k)[i] = 0x88
    q = C.queries(sum(new), 8)
    out, lse = K4.run_attn(cache, q, new, mask)
    s = C.starts(new)
    for p in range(2):
        n, m = cache.lens[p], new[p]
        k, v = cache.rows(p)
        for i in range(m):
            e = C.visible(n - m + i, n, mask)
            bad_k, bad_v = bool(torch.isnan(k[:, :e]).any()), bool(torch.isnan(v[:, :e]).any())
            got = out[s[p] + i].float()
            if bad_k or bad_v:
                assert torch.isnan(got).all()
            else:
                assert torch.isfinite(got).all()
            assert bool(torch.isnan(lse[s[p] + i]).all()) == bad_k and (bad_k or bool(torch.isfinite(lse[s[p] + i]).all()))
    if mask == 0:
        return
    # the rows that see none of them are what they are without them
    clean = K4.filled([200, 90], 8, 2, 16, seed=11)
    ref, _ = K4.run_attn(clean, q, new, mask)
    ok = torch.isfinite(out.float()).all(-1).all(-1)
    assert ok.any() or mask == 32 or max(new) < 4                       # (of few tokens all stand behind such a row)
    assert torch.equal(out[ok], ref[ok])


@pytest.mark.parametrize("heads", [(8, 2), (4, 4), (16, 2)])
def test_rows_of_nan_behind_some_of_few_rows(heads):
    """Two and three tokens, the last of each NaN in its keys and values: the ones before it do not notice."""
    lens, new = [200, 90], [2, 3]
    cache, clean = K4.filled(lens, *heads, 16, seed=11), K4.filled(lens, *heads, 16, seed=11)
    for p in range(2):
        i = cache.at(p, torch.tensor([lens[p] - 1]))
        cache.vs[i] = cache.ks[i] = 255
        cache.v[i] = cache.k[i] = 0x88
    q = C.queries(sum(new), heads[0])
    out, _ = K4.run_attn(cache, q, new, 1)
    assert torch.isnan(out[[1, 4]].float()).all() and torch.isfinite(out[[0, 2, 3]].float()).all()
    for p, rows in ((0, [0]), (1, [2, 3])):
        w, mag, _ = C.attend(clean, p, q[C.starts(new)[p]:C.starts(new)[p + 1]], 1)
        a = C.starts(new)[p]
        for r in rows:
            assert ((out[r].double() - w[r - a]).abs() <= C.OUT_REL * w[r - a].abs() + C.W_REL * mag[r - a] + C.ABS).all()


@pytest.mark.parametrize("new", [[1, 1, 1], [60, 3, 40]])
def test_bad_pages_and_rows_without_keys(new):
    cache = K4.filled([150, 64, 40], 8, 2, 16, seed=2)
    cache.table[0, 3], cache.table[1, :] = -7, 1000                       # a page of the first, all of the second
    cache.seq_lens[2] = max(1, new[2] - 5)                                # the third has more new tokens than cache (or one)
    cache.lens[2] = int(cache.seq_lens[2])
    q, status = C.queries(sum(new), 8), _status()
    out, lse = K4.run_attn(cache, q, new, 1, status=status)
    assert int(status.item()) == mb.DEV_BAD_PAGE
    s = C.starts(new)
    assert (out[s[1]:s[2]] == 0).all() and (lse[s[1]:s[2]] == float("-inf")).all()
    keep = [j for j in range(150) if not 48 <= j < 64]

    class Without:
        H_q, H_kv, lens = 8, 2, [len(keep)]

        def rows(self, p):
            return [x[:, keep] for x in full]
    cache.table[0, 3] = 0
    full = cache.rows(0)
    if new[0] == 1:
        ref, mag, rl = C.attend(Without(), 0, q[:1], 0)
        assert ((out[:1].double() - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS).all()
        assert ((lse[:1].double() - rl).abs() <= C.LSE_ABS).all()
    else:
        for i in (0, 59):
            e = 150 - 60 + i + 1
            left = [j for j in keep if j < e]

            class Part(Without):
                lens = [len(left)]

                def rows(self, p):
                    return [x[:, left] for x in full]
            ref, mag, rl = C.attend(Part(), 0, q[i:i + 1], 0)
            assert ((out[i:i + 1].double() - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS).all()
            assert ((lse[i:i + 1].double() - rl).abs() <= C.LSE_ABS).all()
    C.check_attn(cache, q, new, 1, out, lse, problems=[2])


@pytest.mark.parametrize("size", [2.0 ** -12, 1.0, 2.0 ** 10])
@pytest.mark.parametrize("new", [[1], [50]])
def test_values_of_any_size(size, new):
    """Values near both ends of the format beside ordinary ones, and steep logits."""
    cache = K4.Cache([500], 8, 2, 64, seed=1)
    g = torch.Generator(device="cuda").manual_seed(9)
    k, v = (torch.randn(500, 2, 128, generator=g, device="cuda") for _ in range(2))
    v = v * size
    v[::7] *= 2.0 ** 5
    v[::5] = 0
    k[::11] *= 20
    cache.put(0, torch.arange(500), k, v)
    q = C.queries(sum(new), 8, spread=3.0)
    out, lse = K4.run_attn(cache, q, new, 1)
    s = C.starts(new)
    ref, mag, rl = C.attend(cache, 0, q, 1)
    # logits reach 3 * 20 * 4 here: 128 fp32 additions of products of up to 2^9 are off by 128 * 2^-24 * 2^9 * 128 ** -0.5 at the worst, 4e-4
    # weights below 2^-96 of a row's largest may be lost: the reference of a part of the keys may lie 2^30 below the part's largest weight, and the
    # factor that joins the parts is 0 where it would be below 2^-126.  That is 500 keys of the largest value at most.
    floor = 500 * 2.0 ** -96 * float(cache.rows(0)[1].abs().max())
    bad = (out.double() - ref).abs() > C.OUT_REL * ref.abs() + (2.0 ** -8 + 2e-3) * mag + floor
    assert not bool(bad.any())
    assert ((lse.double() - rl).abs() <= 1e-3).all()


def test_same_as_the_16_bit_cache_that_is_read_from_it():
    cache = K4.filled([777, 300], 28, 4, 64, seed=8)
    k, v = (torch.zeros(2, 4, 777, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv4_read(cache.kv, k, v)
    kv16 = mb.KVCache(k, v, 28, 1, seq_lens=cache.seq_lens)
    for new in ([1, 1], [200, 300]):
        q = C.queries(sum(new), 28)
        out, _ = K4.run_attn(cache, q, new, 1)
        chunk = mb.ChunkBatch(kv16, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), sum(new), max_len=max(new))
        ref = torch.empty_like(out)
        mb.mage_chunk_attn(kv16, chunk, q, 128 ** -0.5, ref, chunk.new_workspace())
        if max(new) > 16:                                                 # the same kernel behind the same tiles
            assert torch.equal(out, ref)
        else:
            C.check_attn(cache, q, new, 1, ref, None)


def test_a_wait_that_runs_out_is_reported():
    cache = K4.filled([400], 8, 2, 64)
    q, status = C.queries(100, 8), _status()
    cache.kv.c.flags = mb.FLAG_TEST_STALL
    K4.run_attn(cache, q, [100], 1, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) & mb.DEV_TIMEOUT
    cache.kv.c.flags = 0
    out, lse = K4.run_attn(cache, q, [100], 1)
    C.check_attn(cache, q, [100], 1, out, lse)


@pytest.mark.parametrize("mask", [0, 1, 32])
@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("heads,lens,new", [((16, 1), [300], [300]), ((28, 4), [700, 600], [320, 330]), ((8, 2), [2000, 0, 1400], [1100, 0, 700])])
def test_written_out_or_rebuilt(mask, page, heads, lens, new):
    """Prompts with the larger workspace (the cache written out in 16 bits first) and with the smaller: the same, and by the definition."""
    cache = K4.filled(lens, *heads, page, seed=3, n_max=max(lens) + 7)
    q = C.queries(sum(new), heads[0])
    chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), q.shape[0], max_len=max(new))
    small, large = mb.load().mage_chunk_workspace_bytes(cache.kv.at, chunk.at), chunk.workspace_bytes()
    assert large >= small + 2 * len(lens) * heads[1] * cache.n_max * 256
    got = [K4.run_attn(cache, q, new, mask, workspace=torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")) for n in (small, large)]
    C.check_attn(cache, q, new, mask, *got[1])
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("page", [16, 128])
def test_written_out_with_bad_pages_and_rows_of_nan(page):
    new, lens, heads = [520, 530], [900, 530], (8, 2)
    cache = K4.filled(lens, *heads, page, seed=6)
    cache.table[0, 1], cache.table[1, 3] = -1, 10 ** 6
    for p, j in ((0, 700), (1, 527)):
        i = cache.at(p, torch.tensor([j]))
        cache.vs[i] = cache.ks[i] = 255
        cache.v[i] = cache.k[i] = 0x88
    q = C.queries(sum(new), heads[0])
    chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), q.shape[0], max_len=max(new))
    small, large = mb.load().mage_chunk_workspace_bytes(cache.kv.at, chunk.at), chunk.workspace_bytes()
    assert large > small
    got = []
    for n in (small, large):
        status = _status()
        got.append(K4.run_attn(cache, q, new, 1, status=status, workspace=torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")))
        torch.cuda.synchronize()
        assert int(status.item()) == mb.DEV_BAD_PAGE
    for a, b in zip(*got):
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))
    out = got[1][0].float()
    assert torch.isnan(out[520 - 200:520]).all() and torch.isfinite(out[:520 - 200]).all() and torch.isnan(out[-3:]).all() and torch.isfinite(out[520:-3]).all()
    # the last row of the first problem that sees no NaN: all its keys but those of the missing page
    e = 700
    keep = [j for j in range(e) if not page <= j < 2 * page]
    cache.table[0, 1] = 0
    full = cache.rows(0)

    class Part:
        H_q, H_kv, lens = 8, 2, [len(keep)]

        def rows(self, p):
            return [x[:, keep] for x in full]
    ref, mag, _ = C.attend(Part(), 0, q[319:320], 0)
    assert ((out[319:320].double() - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS).all()


def test_offsets_past_32_bits():
    """Pools of more than 2^32 bytes and rows of codes at their far ends."""
    H_kv, page, pages = 8, 64, 140000                                     # 4.6 GB of codes in each pool
    table = torch.tensor([[0, 139999, 131072, 3, 139998]], dtype=torch.int32, device="cuda")
    mk = lambda n: torch.zeros(pages, H_kv, page, n, dtype=torch.uint8, device="cuda")
    k, v, ks, vs = mk(64), mk(64), mk(8), mk(8)
    n = 5 * page
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    kv = mb.Kv4Cache(k, v, ks, vs, 16, seq_lens=lens, block_table=table, N_max=n)
    chunk = mb.ChunkBatch(kv, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    new = torch.randn(n, 2 * H_kv, 128, device="cuda").to(torch.bfloat16)
    mb.mage_append_chunk_kv4(kv, chunk, new[:, :H_kv], new[:, H_kv:])
    ko, vo = (torch.zeros(1, H_kv, n, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv4_read(kv, ko, vo)
    for got, x in ((ko, new[:, :H_kv]), (vo, new[:, H_kv:])):
        c, u = K4.quantise(x)
        assert torch.equal(got[0].transpose(0, 1).double(), K4.values(K4.pack(c).cuda(), u.cuda()))
    k16 = mb.KVCache(ko, vo, 16, 1, seq_lens=lens)
    for m in (1, 40, n):                                                  # decoding, rebuilt in the kernel, written out
        q = C.queries(m, 16)
        part = mb.ChunkBatch(kv, torch.tensor([0, m], dtype=torch.int32, device="cuda"), m)
        out, ref = torch.empty_like(q), torch.empty_like(q)
        mb.mage_chunk_attn_kv4(kv, part, q, 128 ** -0.5, out, part.new_workspace())
        mb.mage_chunk_attn(k16, part, q, 128 ** -0.5, ref, part.new_workspace())
        tol = 4 * C.OUT_REL * ref.double().abs() + 2 * C.W_REL * vo.double().abs().max()
        assert ((out.double() - ref.double()).abs() <= tol).all()


def test_two_streams_at_once():
    """Two calls on streams of their own, a workspace each, beside one another and again: as one by one."""
    caches = [K4.filled([3000, 70], 28, 4, 64, seed=s) for s in (1, 2)]
    for new in ([1, 1], [300, 70]):
        qs = [C.queries(sum(new), 28, seed=s) for s in (5, 6)]
        want = [K4.run_attn(c, q, new, 1)[0] for c, q in zip(caches, qs)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        outs = [torch.full_like(q, 7.0) for q in qs]
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        spaces = [mb.ChunkBatch(c.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), sum(new), max_len=max(new)).new_workspace() for c in caches]
        torch.cuda.synchronize()
        for _ in range(3):
            for c, q, o, w, st in zip(caches, qs, outs, spaces, streams):
                K4.run_attn(c, q, new, 1, lse=False, stream=st, status=status, workspace=w, out=o)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


@pytest.mark.parametrize("page", [32, 256, 1024])
@pytest.mark.parametrize("new", [[1, 2], [40, 30], [700, 300]])
def test_other_page_sizes(page, new):
    cache = K4.filled([1500, 300], 8, 2, page, seed=12, n_max=1600)
    q = C.queries(sum(new), 8)
    out, lse = K4.run_attn(cache, q, new, 1)
    C.check_attn(cache, q, new, 1, out, lse)


@pytest.mark.parametrize("new,workspace", [([1, 1], "large"), ([330, 300], "large"), ([330, 300], "small")])
def test_captured_and_replayed_with_other_lengths(new, workspace):
    """A graph of the attention, replayed after the lengths on the device have changed: as a call of its own."""
    cache = K4.filled([900, 700], 28, 4, 64, seed=13)
    n = sum(new)
    q = C.queries(n, 28)
    chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), n, max_len=max(new))
    size = chunk.workspace_bytes() if workspace == "large" else mb.load().mage_chunk_workspace_bytes(cache.kv.at, chunk.at)
    ws, out = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.full((n, 28, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    call = lambda: mb.mage_chunk_attn_kv4(cache.kv, chunk, q, 128 ** -0.5, out, ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lens in ([900, 700], [345, 301], [900, 0]):
        cache.seq_lens.copy_(torch.tensor(lens))
        cache.lens = lens
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        C.check_attn(cache, q, new, 1, out, None, problems=[p for p in range(2) if lens[p]])
        if lens[1] == 0:
            assert (out[new[0]:] == 0).all()


def test_tokens_of_nobody_and_empty_caches():
    """Rows in front of the first range and behind the last are left alone; problems without tokens, without keys, or with neither."""
    cache = K4.filled([50, 0, 30, 0], 8, 2, 16, seed=14, n_max=64)
    q = C.queries(12, 8)
    for starts in ([2, 4, 4, 7, 9], [3, 3, 3, 3, 3]):
        out = torch.full((12, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((12, 8), 7.0, device="cuda")
        for bound in (3, 12):                                             # few rows, and a bound for many
            chunk = mb.ChunkBatch(cache.kv, torch.tensor(starts, dtype=torch.int32, device="cuda"), 12, max_len=bound)
            mb.mage_chunk_attn_kv4(cache.kv, chunk, q, 128 ** -0.5, out, chunk.new_workspace(), lse=lse)
            torch.cuda.synchronize()
            assert (out[:starts[0]] == 7.0).all() and (out[starts[-1]:] == 7.0).all() and (lse[:starts[0]] == 7.0).all() and (lse[starts[-1]:] == 7.0).all()
            for p in range(4):
                a, b = starts[p], starts[p + 1]
                if a == b:
                    continue
                if cache.lens[p] == 0:
                    assert (out[a:b] == 0).all() and (lse[a:b] == float("-inf")).all()
                else:
                    ref, mag, rl = C.attend(cache, p, q[a:b], 1)
                    assert ((out[a:b].double() - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS).all() and ((lse[a:b].double() - rl).abs() <= C.LSE_ABS).all()


@pytest.mark.parametrize("starts,reported", [([0, 0, 700, 700], 0), ([0, 0, 700, 650], mb.DEV_BAD_CHUNK), ([0, 0, 700, 9000], mb.DEV_BAD_CHUNK), ([5, -2, 700, 700], mb.DEV_BAD_CHUNK)])
@pytest.mark.parametrize("mask", [1, 32, 0])
def test_pages_of_problems_without_new_tokens_are_not_looked_at(starts, reported, mask):
    """Slots of a batch with nothing to do, or whose range is none, may have given their pages back: no report of them with either workspace, and the
    same results for the problem that has tokens."""
    lens = [500, 900, 300]
    cache = K4.filled(lens, 8, 2, 16, seed=21)
    cache.table[0, :] = -1
    cache.table[2, 1:] = 10 ** 6
    q, q_start = C.queries(700, 8), torch.tensor(starts, dtype=torch.int32, device="cuda")
    chunk = mb.ChunkBatch(cache.kv, q_start, 700, max_len=700)
    small, large = mb.load().mage_chunk_workspace_bytes(cache.kv.at, chunk.at), chunk.workspace_bytes()
    assert large > small
    got = []
    for n in (small, large):
        status, out, lse = _status(), torch.full((700, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((700, 8), 7.0, device="cuda")
        mb.mage_chunk_attn_kv4(cache.kv, chunk, q, 128 ** -0.5, out, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), mask_block=mask, lse=lse, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == reported
        got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    if starts != sorted(starts):                                          # (entries that do not ascend: results may be anything)
        return
    ref, mag, rl = C.attend(cache, 1, q, mask)
    assert ((out.double() - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS).all() and ((lse.double() - rl).abs() <= C.LSE_ABS).all()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("heads,m", [((8, 2), 1), ((8, 2), 4)])
@pytest.mark.parametrize("n,missing", [(64, [0]), (64, [1]), (64, [0, 1]), (64, [1, 2, 3]), (64, [0, 2, 3]), (64, [0, 1, 2, 3]), (1100, list(range(68))), (1100, list(range(69))), (1100, [0, 5, 68])])
def test_keys_taken_beside_missing_pages(bits, heads, m, n, missing):
    """Whether a row took a key does not hang on its logits: with no logit above -inf (or NaN ones) it is 0 / 0 where some page is there, and zeros where none is."""
    cache = K4.filled([n], *heads, 16, seed=31) if bits == 4 else C.filled([n], *heads, 16, bits, seed=31)
    x = torch.ones(n, heads[1], 128, device="cuda")
    cache.put(0, torch.arange(n), x, x)
    for j in missing:
        cache.table[0, j] = -1
    q = torch.ones(m, heads[0], 128, device="cuda").to(torch.bfloat16)
    q[:, :, 5] = float("-inf")
    chunk = mb.ChunkBatch(cache.kv, torch.tensor([0, m], dtype=torch.int32, device="cuda"), m)
    out, status = torch.full_like(q, 7.0), _status()
    call = {16: mb.mage_chunk_attn, 8: mb.mage_chunk_attn_kv8, 4: mb.mage_chunk_attn_kv4}[bits]
    call(cache.kv, chunk, q, 128 ** -0.5, out, chunk.new_workspace(), mask_block=0, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == mb.DEV_BAD_PAGE
    if len(missing) * 16 >= n:
        assert (out == 0).all()
    else:
        assert torch.isnan(out).all()


@pytest.mark.parametrize("tokens,large,waits", [(1, True, False), (5, True, False), (8, True, False), (9, True, True), (200, False, True), (200, True, True)])
def test_which_calls_have_waits_that_can_run_out(tokens, large, waits):
    """The flag that holds back the first key tile: up to 32 rows per KV head (four a token here) nothing waits for it; above, over the copy or over codes, the wait is reported."""
    cache = K4.filled([400], 8, 2, 64, seed=15)
    q, status = C.queries(tokens, 8), _status()
    chunk = mb.ChunkBatch(cache.kv, torch.tensor([0, tokens], dtype=torch.int32, device="cuda"), tokens)
    small = mb.load().mage_chunk_workspace_bytes(cache.kv.at, chunk.at)
    assert (chunk.workspace_bytes() > small) == (tokens == 200)
    ws = torch.empty(chunk.workspace_bytes() if large else small, dtype=torch.uint8, device="cuda")
    cache.kv.c.flags = mb.FLAG_TEST_STALL
    out, lse = K4.run_attn(cache, q, [tokens], 1, status=status, workspace=ws)
    torch.cuda.synchronize()
    assert int(status.item()) == (mb.DEV_TIMEOUT if waits else 0)
    cache.kv.c.flags = 0
    if waits:
        out, lse = K4.run_attn(cache, q, [tokens], 1, workspace=ws)
    C.check_attn(cache, q, [tokens], 1, out, lse)
