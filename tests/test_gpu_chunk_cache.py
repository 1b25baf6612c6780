"""Rotary positions, cache writes in 16 and 8 bits, the 8-bit cache read back, and the calls in a row as a server makes them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import chunk_harness as C
from paper_2602_14209_b200 import binding as mb


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("n", [1, 2, 5, 333, 1500])
@pytest.mark.parametrize("rot,halves", [(128, True), (128, False), (64, True), (96, True), (16, False), (48, False)])
@pytest.mark.parametrize("H_q,H_kv,axes", [(28, 4, 3), (3, 3, 1), (5, 1, 4)])
def test_rope(n, rot, halves, H_q, H_kv, axes):
    """y = mult (x1 cos - x2 sin): fp32 products and sums (2^-22 of |x1| + |x2|), then half a bf16 step."""
    g = torch.Generator().manual_seed(n + rot)
    pairs = rot // 2
    pos = torch.randint(-1000, 2 ** 31 - 1 if n == 5 else 2 * 10 ** 6, (axes, n), generator=g, dtype=torch.int64).int()
    inv = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float()
    axis = torch.randint(0, axes, (pairs,), generator=g)
    axis[0] = axes - 1
    big = torch.randn(n, H_q + 2 * H_kv, 128, generator=g).to(torch.bfloat16).cuda()
    q, k = big[:, :H_q], big[:, H_q:H_q + H_kv]
    rope = mb.Rope(inv.cuda(), axis_of_pair=axis.tolist(), rot_dim=rot, halves=halves, mult=1.25)
    qo, ko = torch.empty(n, H_q, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(n, H_kv, 128, dtype=torch.bfloat16, device="cuda")
    mb.mage_rope(rope, pos.cuda(), q, k, qo, ko)
    import numpy as np
    turn = pos.double().numpy()[axis.numpy()].T.astype(np.longdouble) * inv.double().numpy().astype(np.longdouble)
    turn = np.fmod(turn, 2 * np.arctan2(np.longdouble(0), np.longdouble(-1)))
    c, s = torch.from_numpy(np.cos(turn).astype(np.float64))[:, None], torch.from_numpy(np.sin(turn).astype(np.float64))[:, None]
    for x, y in ((q, qo), (k, ko)):
        x, y = x.double().cpu(), y.double().cpu()
        lo, hi = (slice(0, pairs), slice(pairs, rot)) if halves else (slice(0, rot, 2), slice(1, rot, 2))
        ref, tol = x.clone(), torch.zeros_like(x)
        ref[..., lo] = 1.25 * (x[..., lo] * c - x[..., hi] * s)
        ref[..., hi] = 1.25 * (x[..., hi] * c + x[..., lo] * s)
        size = (x[..., lo].abs() + x[..., hi].abs()) * 1.25
        # angle: 2^-52 of up to 2^31 turns, then the fraction in single precision: below 2e-6 for the far ones, 2^-22 else
        d = 2e-6 if n == 5 else 2.0 ** -21
        tol[..., lo] = tol[..., hi] = size * d
        assert ((y - ref).abs() <= tol + ref.abs() * 2.0 ** -8 * (rot and 1)).all()
        assert torch.equal(y[..., rot:], x[..., rot:])
    # in place gives the same bits, and leaves the values beside them alone
    before = big.clone()
    mb.mage_rope(rope, pos.cuda(), q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(big[:, H_q + H_kv:], before[:, H_q + H_kv:])
    mb.mage_rope(rope, pos.cuda(), before[:, :H_q], None, qo.zero_())
    assert torch.equal(qo, q)


def _append(cache, new, k, v, status=None, max_len=None):
    chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), k.shape[0], max_len=max(new) if max_len is None else max_len)
    (mb.mage_append_chunk if cache.bits == 16 else mb.mage_append_chunk_kv8)(cache.kv, chunk, k, v, dev_status=status)


def _pools(c):
    return [c.k, c.v] if c.bits == 16 else [c.k, c.v, c.ks, c.vs]


def _same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("H_kv", [1, 2, 5, 8])
@pytest.mark.parametrize("new,ctx", [([1], [0]), ([1, 1, 1], [0, 63, 200]), ([3, 0, 70, 1], [0, 4, 60, 15]), ([600, 900], [31, 0])])
def test_append_writes_its_rows_and_nothing_else(bits, page, H_kv, new, ctx):
    lens = [c + m for c, m in zip(ctx, new)]
    cache, want = (C.Cache(lens, H_kv, H_kv, page, bits, n_max=max(lens) + 40) for _ in range(2))
    n = sum(new) + 3
    g = torch.Generator().manual_seed(n)
    scale = torch.exp(torch.randn(n, 1, 1, generator=g) * 8)                 # magnitudes over twenty binades
    big = (torch.randn(n, 3 * H_kv, 128, generator=g) * scale).to(torch.bfloat16).cuda()
    k, v = big[:, H_kv:2 * H_kv], big[:, 2 * H_kv:]
    v[0, 0] = 0                                                             # an all-zero row: scale 1
    k[-4, -1, 7] = float("inf")
    status = _status()
    _append(cache, new, k, v, status)
    s = C.starts(new)
    for p, m in enumerate(new):
        if m:
            want.put(p, ctx[p] + torch.arange(m), k[s[p]:s[p + 1]], v[s[p]:s[p + 1]])
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for a, b in zip(_pools(cache), _pools(want)):
        if a.dtype == torch.float32:
            assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(-1), b.nan_to_num(-1))
        else:
            assert _same_bits(a, b)


def test_quantised_codes_are_those_of_the_division():
    """Every bf16 magnitude of some binades against every kind of row maximum: the quotient is the correctly rounded one."""
    n = 4096
    g = torch.Generator().manual_seed(0)
    bits = torch.randint(0, 2 ** 15, (n, 1, 128), generator=g).to(torch.int16)
    x = bits.view(torch.bfloat16)
    x = torch.where(torch.isfinite(x), x, torch.ones_like(x))
    near = torch.randn(n, 1, 128, generator=g).to(torch.bfloat16)            # ordinary rows
    edge = (torch.arange(n * 128).view(n, 1, 128) % 449).to(torch.bfloat16) * torch.exp2(torch.randint(-120, 110, (n, 1, 1), generator=g).float()).to(torch.bfloat16)
    for rows in (x, near, edge, x * 2.0 ** -100):
        cache = C.Cache([n], 1, 1, 0, 8)
        _append(cache, [n], rows.cuda(), rows.cuda().clone())
        code, s = C.quantise(rows)
        assert torch.equal(cache.ks[0, 0].cpu(), s[:, 0])
        assert torch.equal(cache.k[0, 0].cpu(), code[:, 0].view(torch.uint8))


def test_append_refuses_what_does_not_fit():
    new = [4, 2, 3]
    for bits in (16, 8):
        cache, want = (C.Cache([10, 1, 40], 2, 2, 16, bits) for _ in range(2))
        cache.seq_lens[2] = 50                                               # problem 1: fewer rows than new tokens; 2: beyond N_max
        k = C.queries(sum(new), 2)
        status = _status()
        _append(cache, new, k, k, status)
        torch.cuda.synchronize()
        assert int(status.item()) == mb.DEV_CACHE_FULL
        want.put(0, 6 + torch.arange(4), k[:4], k[:4])
        assert all(_same_bits(a, b) for a, b in zip(_pools(cache), _pools(want)))
        cache = C.Cache([10, 20, 30], 2, 2, 16, bits)
        cache.table[1, 1] = -5
        status.zero_()
        _append(cache, [4, 8, 3], C.queries(15, 2), C.queries(15, 2), status)
        torch.cuda.synchronize()
        assert int(status.item()) == mb.DEV_BAD_PAGE


@pytest.mark.parametrize("page", [0, 32])
def test_read_back(page):
    lens = [0, 1, 70, 333]
    cache = C.filled(lens, 6, 3, page, 8, n_max=400)
    g = torch.Generator().manual_seed(1)
    for begin, n in ((0, 400), (0, 1), (69, 7), (300, 100)):
        ko, vo = (torch.full((4, 3, n, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        status = _status()
        mb.mage_kv8_read(cache.kv, ko, vo, row_begin=begin, dev_status=status)
        for p, m in enumerate(lens):
            k, v = cache.rows(p)
            got = max(0, min(m - begin, n))
            for o, x in ((ko, k), (vo, v)):
                assert torch.equal(o[p, :, :got], x[:, begin:begin + got].float().to(torch.bfloat16))
                assert (o[p, :, got:] == 7.0).all()
        assert int(status.item()) == 0
    k_sel = 50
    idx = torch.full((4, 3, k_sel), -1, dtype=torch.int32)
    for p, m in enumerate(lens):
        for h in range(3):
            idx[p, h, :min(m, k_sel)] = torch.randperm(m, generator=g)[:k_sel].sort().values.int()
    idx[3, 1, 4] = 333                                                      # outside: reported, left as it was
    keff = torch.tensor([min(m, k_sel) for m in lens], dtype=torch.int32).cuda()
    ko, vo = (torch.full((4, 3, k_sel, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    status = _status()
    mb.mage_kv8_read(cache.kv, ko, vo, indices=idx.cuda(), k_eff=keff, dev_status=status)
    assert int(status.item()) == mb.DEV_BAD_INDEX
    for p, m in enumerate(lens):
        k, v = cache.rows(p)
        for h in range(3):
            for t in range(k_sel):
                j = int(idx[p, h, t])
                for o, x in ((ko, k), (vo, v)):
                    want = x[h, j].float().to(torch.bfloat16) if 0 <= j < m else torch.full((128,), 7.0, dtype=torch.bfloat16, device="cuda")
                    assert torch.equal(o[p, h, t], want)


def test_prompt_in_chunks_then_blocks_over_the_8_bit_cache():
    """A server's round: rotate, write to the 8-bit cache, attend -- a prompt in three ragged chunks and two decoded tokens -- then
    the prefix read back for the exact pass and the selection, the selected rows read back for a reuse step."""
    H_q, H_kv, page, P, B, k_sel = 28, 4, 64, 3, 32, 64
    steps = [[100, 33, 7], [40, 0, 64], [1, 200, 1], [1, 1, 1], [1, 1, 1]]
    total = [sum(s[p] for s in steps) for p in range(P)]
    cache = C.Cache(total, H_q, H_kv, page, 8)
    cache.lens = [0] * P
    cache.seq_lens.zero_()
    inv = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    rope = mb.Rope(inv, axis_of_pair=[0] * 24 + [1] * 20 + [2] * 20)
    for i, new in enumerate(steps):
        n = sum(new)
        qkv = C.queries(n, H_q + 2 * H_kv, seed=20 + i)
        pos = torch.cat([torch.arange(cache.lens[p], cache.lens[p] + m) for p, m in enumerate(new)]).int().cuda().expand(3, n).contiguous()
        cache.lens = [a + b for a, b in zip(cache.lens, new)]
        cache.seq_lens.copy_(torch.tensor(cache.lens, dtype=torch.int32))
        chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), n, max_len=max(new))
        q, k, v = qkv[:, :H_q], qkv[:, H_q:H_q + H_kv], qkv[:, H_q + H_kv:]
        status = _status()
        mb.mage_rope(rope, pos, q, k)
        mb.mage_append_chunk_kv8(cache.kv, chunk, k, v, dev_status=status)
        out, lse = torch.full((n, H_q, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((n, H_q), 7.0, device="cuda")
        mb.mage_chunk_attn_kv8(cache.kv, chunk, q, 128 ** -0.5, out, chunk.new_workspace(), mask_block=1, lse=lse, dev_status=status)
        assert int(status.item()) == 0
        C.check_attn(cache, q, new, 1, out, lse)
        # what was written is what the definition writes
        s = C.starts(new)
        for p, m in enumerate(new):
            code, sc = C.quantise(k[s[p]:s[p + 1]])
            i_ = cache.at(p, torch.arange(cache.lens[p] - m, cache.lens[p]))
            assert torch.equal(cache.k[i_].cpu(), code.view(torch.uint8)) and torch.equal(cache.ks[i_].cpu(), sc)
    # the prefix as a 16-bit cache: exact pass and selection of a block
    n_max = max(cache.lens)
    kr, vr = (torch.zeros(P, H_kv, n_max, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv8_read(cache.kv, kr, vr)
    kv = mb.KVCache(kr, vr, H_q, B, seq_lens=cache.seq_lens)
    from paper_2602_14209_b200.pipeline import BlockAttention
    ba = BlockAttention(kv, k_sel)
    q, kb, vb = (C.queries(P * B, h, seed=50 + h).view(P, B, h, 128).transpose(1, 2).contiguous() for h in (H_q, H_kv, H_kv))
    ba.exact_select(q, kb, vb)
    ba.select_async()
    ba.join()
    ref = ba.sparse_step(q, kb, vb).clone()
    # the reuse step over the selected rows alone, read back from the 8-bit cache
    ks, vs = (torch.zeros(P, H_kv, k_sel, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv8_read(cache.kv, ks, vs, indices=ba.indices, k_eff=ba.k_eff)
    small = mb.KVCache(ks, vs, H_q, B, seq_lens=ba.k_eff)
    every = torch.arange(k_sel, dtype=torch.int32, device="cuda").expand(P, H_kv, k_sel).contiguous()
    got = torch.empty_like(ref)
    mb.mage_sparse_block_attn(small, q, kb, vb, every, ba.k_eff, k_sel, 128 ** -0.5, got, small.new_workspace(k_sel))
    torch.cuda.synchronize()
    assert torch.equal(got, ref)


def test_16_bit_chunks_feed_the_block_path():
    """mage_append_chunk over a paged 16-bit cache, then a block's exact pass over it."""
    H_q, H_kv, lens = 8, 2, [130, 64]
    cache = C.Cache(lens, H_q, H_kv, 64, 16)
    k, v = C.queries(sum(lens), H_kv, seed=1), C.queries(sum(lens), H_kv, seed=2)
    _append(cache, lens, k, v)
    want = C.Cache(lens, H_q, H_kv, 64, 16)
    for p, (a, b) in enumerate(((0, 130), (130, 194))):
        want.put(p, torch.arange(lens[p]), k[a:b], v[a:b])
    assert all(_same_bits(x, y) for x, y in zip(_pools(cache), _pools(want)))
    q, kb, vb = (C.queries(2 * 16, h, seed=5).view(2, 16, h, 128).transpose(1, 2).contiguous() for h in (H_q, H_kv, H_kv))
    outs = []
    for c in (cache, want):
        kv = mb.KVCache(c.k, c.v, H_q, 16, seq_lens=c.seq_lens, block_table=c.table, N_max=130)
        o = torch.empty(2, H_q, 16, 128, dtype=torch.bfloat16, device="cuda")
        mb.mage_exact_attn(kv, q, kb, vb, 128 ** -0.5, o, kv.new_workspace())
        outs.append(o)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and torch.isfinite(outs[0]).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_append_reports_ranges_that_are_none(bits):
    """q_start that does not ascend: the problem with the empty range is reported though no token falls into it."""
    cache = C.Cache([10, 20, 30], 2, 2, 16, bits)
    x = torch.randn(12, 2, 128, device="cuda").to(torch.bfloat16)
    status = _status()
    chunk = mb.ChunkBatch(cache.kv, torch.tensor([0, 8, 4, 12], dtype=torch.int32, device="cuda"), 12, max_len=8)
    (mb.mage_append_chunk if bits == 16 else mb.mage_append_chunk_kv8)(cache.kv, chunk, x, x, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == mb.DEV_BAD_CHUNK
