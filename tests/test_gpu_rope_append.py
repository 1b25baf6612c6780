"""Cache writes that rotate on the way, against the rotation's definition in 64 bits and the formats' own."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import chunk_harness as C
import kv4_harness as K4
from paper_2602_14209_b200 import binding as mb

CALLS = {16: "mage_rope_append_chunk", 8: "mage_rope_append_chunk_kv8", 4: "mage_rope_append_chunk_kv4"}


def _cache(bits, lens, H_q, H_kv, page, **kw):
    return K4.Cache(lens, H_q, H_kv, page, **kw) if bits == 4 else C.Cache(lens, H_q, H_kv, page, bits, **kw)


def _pools(c):
    return [x.clone() for x in ((c.k, c.v) if c.bits == 16 else (c.k, c.v, c.ks, c.vs))]


def _bits(x):
    return x.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()])


def _same(a, b):
    return torch.equal(_bits(a), _bits(b))


def _rope(rot, halves, axes, seed=0, mult=1.0):
    pairs = rot // 2
    g = torch.Generator().manual_seed(seed)
    inv = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float()
    axis = torch.randint(0, axes, (pairs,), generator=g)
    axis[0] = axes - 1
    return mb.Rope(inv.cuda(), axis_of_pair=axis.tolist(), rot_dim=rot, halves=halves, mult=mult), inv, axis


def _turned(x, pos, inv, axis, rot, halves, mult):
    """(rotated x in 64 bits, bound of the fp32 arithmetic's error): as for the rotation alone."""
    turn = pos.double()[axis].T * inv.double()
    c, s = turn.cos()[:, None], turn.sin()[:, None]
    x = x.double().cpu()
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if halves else (slice(0, rot, 2), slice(1, rot, 2))
    y, tol = x.clone(), torch.zeros_like(x)
    y[..., lo], y[..., hi] = mult * (x[..., lo] * c - x[..., hi] * s), mult * (x[..., hi] * c + x[..., lo] * s)
    tol[..., lo] = tol[..., hi] = (x[..., lo].abs() + x[..., hi].abs()) * mult * 2.0 ** -21
    return y, tol


def _call(cache, new, rope, pos, q, k, v, q_out=None, status=None, n_tokens=None, max_len=None, stream=None):
    chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), q.shape[0], max_len=max(new) if max_len is None else max_len)
    getattr(mb, CALLS[cache.bits])(cache.kv, chunk, rope, pos, q, k, v, q_out=q_out, dev_status=status, stream=stream)


@pytest.mark.parametrize("rot,halves", [(128, True), (128, False), (64, True), (80, True), (96, False), (16, True)])
@pytest.mark.parametrize("H_q,H_kv,axes", [(28, 4, 3), (3, 3, 1), (5, 1, 4), (16, 8, 2)])
@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("new", [[1, 1, 1], [5, 0, 40], [700, 3, 600]])
def test_rotated_and_written(rot, halves, H_q, H_kv, axes, page, new):
    ctx = [7, 0, 64]
    lens, n, s = [c + m for c, m in zip(ctx, new)], sum(new), C.starts(new)
    g = torch.Generator().manual_seed(n + rot)
    big = torch.randn(n, H_q + 2 * H_kv, 128, generator=g).to(torch.bfloat16).cuda()
    q, k, v = big[:, :H_q], big[:, H_q:H_q + H_kv], big[:, H_q + H_kv:]
    pos = torch.randint(-1000, 10 ** 6, (axes, n), generator=g, dtype=torch.int64).int()
    rope, inv, axis = _rope(rot, halves, axes, n, 1.25)
    kept, rows = big.clone(), {}
    for bits in (16, 8, 4):
        cache = _cache(bits, lens, H_q, H_kv, page, n_max=800, seed=3)
        before, q_out, status = _pools(cache), torch.empty(n, H_q, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        _call(cache, new, rope, pos.cuda(), q, k, v, q_out, status)
        assert int(status.item()) == 0 and torch.equal(big, kept)
        y, tol = _turned(q, pos, inv, axis, rot, halves, 1.25)
        assert ((q_out.double().cpu() - y).abs() <= tol + y.abs() * 2.0 ** -8).all() and torch.equal(q_out[..., rot:], q[..., rot:])
        for p, m in enumerate(new):
            if m == 0:
                continue
            i = cache.at(p, torch.arange(ctx[p], ctx[p] + m))
            swap = (lambda x: x) if page else (lambda x: x.transpose(0, 1))
            if bits == 16:
                got = swap(cache.k[i])
                yk, tk = _turned(k[s[p]:s[p + 1]], pos[:, s[p]:s[p + 1]], inv, axis, rot, halves, 1.25)
                assert ((got.double().cpu() - yk).abs() <= tk + yk.abs() * 2.0 ** -8).all() and torch.equal(got[..., rot:], k[s[p]:s[p + 1], :, rot:])
                rows[p] = got
                before[0][i], before[1][i] = cache.k[i], swap(v[s[p]:s[p + 1]])
            else:                                          # the same rows, coded from their bf16 values
                for which, x in ((0, rows[p]), (1, v[s[p]:s[p + 1]])):
                    if bits == 8:
                        c, sc = C.quantise(x)
                        c = c.view(torch.uint8)
                    else:
                        c, sc = K4.quantise(x)
                        c = K4.pack(c)
                    before[which][i], before[2 + which][i] = swap(c).cuda(), swap(sc).cuda()
        for got, want in zip(_pools(cache), before):       # and no other row
            assert _same(got, want)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("n", [3, 1400])
def test_queries_like_the_rotation_alone(bits, n):
    rope, _, _ = _rope(128, True, 3)
    big = torch.randn(n, 28 + 8, 128, device="cuda").to(torch.bfloat16)
    q, k, v = big[:, :28], big[:, 28:32], big[:, 32:]
    pos = torch.randint(0, 100000, (3, n), dtype=torch.int32, device="cuda")
    want = torch.empty(n, 28, 128, dtype=torch.bfloat16, device="cuda")
    mb.mage_rope(rope, pos, q, None, want)
    cache = _cache(bits, [n], 28, 4, 64)
    _call(cache, [n], rope, pos, q, k, v)                  # in place
    assert torch.equal(q, want)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_tokens_without_a_place(bits):
    """Nobody's tokens, ranges that are none, caches that are full, bad pages."""
    cache = _cache(bits, [40, 20, 9, 12], 4, 2, 16, n_max=48)
    cache.seq_lens.copy_(torch.tensor([49, 20, 3, 12]))             # too long, fine, shorter than its new tokens, fine
    cache.table[1, 1] = 99
    before, status = _pools(cache), torch.zeros(1, dtype=torch.int32, device="cuda")
    rope, _, _ = _rope(64, True, 1)
    n = 20
    q, k = torch.randn(n, 4, 128, device="cuda").to(torch.bfloat16), torch.randn(n, 2, 128, device="cuda").to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    want = torch.empty_like(q)
    mb.mage_rope(rope, pos, q, None, want)
    out = torch.full_like(q, 7.0)
    chunk = mb.ChunkBatch(cache.kv, torch.tensor([1, 5, 11, 15, 17], dtype=torch.int32, device="cuda"), n, max_len=6)
    getattr(mb, CALLS[bits])(cache.kv, chunk, rope, pos, q, k, k, q_out=out, dev_status=status)
    assert int(status.item()) == mb.DEV_CACHE_FULL | mb.DEV_BAD_PAGE
    assert torch.equal(out[1:17], want[1:17]) and (out[:1] == 7.0).all() and (out[17:] == 7.0).all()
    changed = [tuple(i) for pool, old in zip(_pools(cache), before) for i in (_bits(pool) != _bits(old)).nonzero()[:, [0, 2]].unique(dim=0).tolist()]      # (page, row)
    ok = {(int(cache.table[1, 0]), 14), (int(cache.table[1, 0]), 15), (int(cache.table[3, 0]), 10), (int(cache.table[3, 0]), 11)}
    assert set(changed) <= ok and len(set(changed)) == 4
    status.zero_()
    out.fill_(7.0)
    chunk = mb.ChunkBatch(cache.kv, torch.tensor([0, 9, 4, 4, 99], dtype=torch.int32, device="cuda"), n, max_len=6)
    after = _pools(cache)
    getattr(mb, CALLS[bits])(cache.kv, chunk, rope, pos, q, k, k, q_out=out, dev_status=status)
    assert int(status.item()) & mb.DEV_BAD_CHUNK and (out == 7.0).all()
    for pool, old in zip(_pools(cache), after):
        assert _same(pool, old)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [[1, 1, 1], [33, 1, 64]])
def test_a_layer_as_a_server_runs_it(bits, new):
    """Rotate, write, attend, in one captured graph on a stream of its own, replayed with new tokens: as the calls one by one."""
    H_q, H_kv, page, ctx = 28, 4, 64, [300, 5, 129]
    lens, n = [c + m for c, m in zip(ctx, new)], sum(new)
    cache = (K4.filled(lens, H_q, H_kv, page) if bits == 4 else C.filled(lens, H_q, H_kv, page, bits))
    rope, _, _ = _rope(128, True, 1)
    pos = torch.cat([torch.arange(c, c + m) for c, m in zip(ctx, new)]).int().cuda()
    qkv = torch.randn(n, H_q + 2 * H_kv, 128, device="cuda").to(torch.bfloat16)
    q_start = torch.tensor(C.starts(new), dtype=torch.int32, device="cuda")
    chunk = mb.ChunkBatch(cache.kv, q_start, n, max_len=max(new))
    ws, q_out, out = chunk.new_workspace(), torch.empty(n, H_q, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(n, H_q, 128, dtype=torch.bfloat16, device="cuda")
    attn = {16: mb.mage_chunk_attn, 8: mb.mage_chunk_attn_kv8, 4: mb.mage_chunk_attn_kv4}[bits]

    def layer():
        getattr(mb, CALLS[bits])(cache.kv, chunk, rope, pos, qkv[:, :H_q], qkv[:, H_q:H_q + H_kv], qkv[:, H_q + H_kv:], q_out=q_out)
        attn(cache.kv, chunk, q_out, 128 ** -0.5, out, ws, mask_block=1)

    layer()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        layer()
    for seed in (1, 2):
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        C_out = got.double()
        for p, m in enumerate(new):
            a = C.starts(new)[p]
            ref, mag, _ = C.attend(cache, p, q_out[a:a + m], 1)
            assert ((C_out[a:a + m] - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS).all()
        layer()
        torch.cuda.synchronize()
        assert torch.equal(out, got)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_one_head_and_many(bits):
    """One query head, one KV head; and head counts that no step of the kernel divides."""
    for H_q, H_kv, n in ((1, 1, 1500), (1, 1, 2), (33, 11, 1301), (33, 11, 3)):
        rope, inv, axis = _rope(128, True, 1)
        x = torch.randn(n, H_q + 2 * H_kv, 128, device="cuda").to(torch.bfloat16)
        pos = torch.arange(n, dtype=torch.int32, device="cuda")
        cache, plain = (_cache(bits, [n], H_q, H_kv, 16) for _ in range(2))
        q, k = torch.empty(n, H_q, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(n, H_kv, 128, dtype=torch.bfloat16, device="cuda")
        _call(cache, [n], rope, pos, x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:], q)
        want = torch.empty_like(q)
        mb.mage_rope(rope, pos, x[:, :H_q], x[:, H_q:H_q + H_kv], want, k)
        assert torch.equal(q, want)
        chunk = mb.ChunkBatch(plain.kv, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
        v = x[:, H_q + H_kv:].contiguous()
        {16: mb.mage_append_chunk, 8: mb.mage_append_chunk_kv8, 4: mb.mage_append_chunk_kv4}[bits](plain.kv, chunk, k, v)
        for a, b in zip(_pools(cache), _pools(plain)):                    # the rotation and the write one after the other
            assert _same(a, b)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("rot,halves", [(128, True), (128, False), (80, True), (80, False), (16, True), (16, False)])
@pytest.mark.parametrize("n,mult", [(3, 1.25), (1300, 1.25), (1300, 1.0)])
def test_as_the_rotation_and_the_write_one_after_the_other(bits, rot, halves, n, mult):
    """Queries, codes and scales, bit for bit, in every form of the rotation: infinities and NaN among the new tokens as well."""
    H_q, H_kv = 6, 3
    rope, _, _ = _rope(rot, halves, 2, rot, mult)
    g = torch.Generator().manual_seed(n + rot)
    x = torch.randn(n, H_q + 2 * H_kv, 128, generator=g)
    x[torch.rand(x.shape, generator=g) < 2.0 ** -12] = float("nan")
    x[torch.rand(x.shape, generator=g) < 2.0 ** -12] = float("inf")
    x[torch.rand(x.shape, generator=g) < 2.0 ** -12] = float("-inf")
    x = x.to(torch.bfloat16).cuda()
    pos = torch.randint(-10 ** 6, 10 ** 6, (2, n), generator=g, dtype=torch.int64).int().cuda()
    cache, plain = (_cache(bits, [n], H_q, H_kv, 16) for _ in range(2))
    q, want = (torch.empty(n, H_q, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k = torch.empty(n, H_kv, 128, dtype=torch.bfloat16, device="cuda")
    _call(cache, [n], rope, pos, x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:], q)
    mb.mage_rope(rope, pos, x[:, :H_q], x[:, H_q:H_q + H_kv], want, k)
    chunk = mb.ChunkBatch(plain.kv, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    {16: mb.mage_append_chunk, 8: mb.mage_append_chunk_kv8, 4: mb.mage_append_chunk_kv4}[bits](plain.kv, chunk, k, x[:, H_q + H_kv:].contiguous())
    for a, b in zip([q] + _pools(cache), [want] + _pools(plain)):
        assert torch.equal(torch.isnan(a), torch.isnan(b)) if a.is_floating_point() else True
        assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) if a.is_floating_point() else torch.equal(a, b)
