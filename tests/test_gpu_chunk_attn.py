"""mage_chunk_attn / mage_chunk_attn_kv8 against the definition in 64 bits: single tokens to long chunks, ragged and empty problems,
both cache types, pages that end inside a tile, masks, NaN patterns everywhere a row does not look, split and unsplit runs."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

import chunk_harness as C
from paper_2602_14209_b200 import binding as mb

BITS = pytest.mark.parametrize("bits", [16, 8])


@BITS
@pytest.mark.parametrize("page", [0, 16, 64, 256])
@pytest.mark.parametrize("H_q,H_kv", [(8, 2), (28, 4), (3, 3), (40, 2), (32, 1)])
def test_single_tokens_over_ragged_prefixes(bits, page, H_q, H_kv):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 2049]
    cache = C.filled(lens, H_q, H_kv, page, bits, seed=H_q + page)
    q = C.queries(len(lens), H_q)
    out, lse = C.run_attn(cache, q, [1] * len(lens), 1)
    C.check_attn(cache, q, [1] * len(lens), 1, out, lse)


@BITS
@pytest.mark.parametrize("mask", [0, 1, 7, 32])
@pytest.mark.parametrize("H_q,H_kv,page", [(8, 2, 64), (28, 4, 16), (5, 1, 0), (2, 2, 32)])
def test_chunks_of_odd_lengths(bits, mask, H_q, H_kv, page):
    new = [3, 0, 1, 130, 65, 1, 0, 31, 257, 2]
    ctx = [0, 5, 0, 0, 700, 1000, 0, 33, 511, 4000]
    lens = [c + m for c, m in zip(ctx, new)]
    cache = C.filled(lens, H_q, H_kv, page, bits, seed=mask)
    q = C.queries(sum(new) + 5, H_q)
    out, lse = C.run_attn(cache, q, new, mask)
    C.check_attn(cache, q, new, mask, out, lse)


@BITS
@pytest.mark.parametrize("new", [[1], [2], [9], [40], [300]])
@pytest.mark.parametrize("n", [1, 100, 129, 5000])
def test_one_problem_split_over_many_blocks(bits, new, n):
    lens = [max(n, new[0])]
    cache = C.filled(lens, 8, 2, 64, bits, seed=n)
    q = C.queries(new[0], 8)
    for mask in (0, 1):
        out, lse = C.run_attn(cache, q, new, mask)
        C.check_attn(cache, q, new, mask, out, lse)


@BITS
def test_many_problems(bits):
    """More problems than threads in a block, most of them tiny."""
    g = torch.Generator().manual_seed(5)
    lens = (torch.rand(700, generator=g) ** 6 * 3000).int().add(1).tolist()
    new = [1 if i % 3 else 0 for i in range(700)]
    cache = C.filled(lens, 4, 1, 16, bits, seed=1)
    q = C.queries(sum(new), 4)
    out, lse = C.run_attn(cache, q, new, 1)
    C.check_attn(cache, q, new, 1, out, lse, problems=range(0, 700, 7))


@BITS
def test_rows_that_see_nothing(bits):
    """More new tokens than the length: positions below zero.  And a problem of length zero."""
    lens, new = [0, 2, 200], [3, 5, 4]
    cache = C.filled(lens, 8, 2, 64, bits, n_max=256)
    q = C.queries(sum(new), 8)
    out, lse = C.run_attn(cache, q, new, 1)
    C.check_attn(cache, q, new, 1, out, lse)
    assert (out[:3] == 0).all() and torch.isinf(lse[:3]).all() and (out[3:6] == 0).all()


@BITS
@pytest.mark.parametrize("m", [4, 150, 400])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_keys_and_values_behind_the_mask_may_be_anything(bits, m, bad):
    """Tokens whose keys or values are NaN or infinite: rows that do not see them are as without them; rows that do see what the
    definition gives (an 8-bit row with such an element is NaN as a whole)."""
    n = m + 300
    cache = C.filled([n], 8, 2, 64, bits)
    q = C.queries(m, 8)
    for row, what in ((n - m + m // 3, "v"), (n - m + m // 2, "k"), (n - 1, "v")):
        k, v = (torch.randn(1, 2, 128) for _ in range(2))
        (v if what == "v" else k)[0, :, 5] = bad
        cache.put(0, torch.tensor([row]), k, v)
    out, lse = C.run_attn(cache, q, [m], 1)
    first_k = m // 2                                        # rows in front of the bad key: by the definition
    ref, mag, rl = C.attend(cache, 0, q, 1)
    got = out.double()
    fin = torch.isfinite(ref[:first_k])
    assert torch.equal(torch.isfinite(got[:first_k]), fin)
    assert ((got - ref)[:first_k][fin].abs() <= (C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS)[:first_k][fin]).all()
    assert torch.isfinite(got[:m // 3]).all()
    if bad == bad and bits == 16:                           # an infinite value: its sign where rows see it
        assert torch.equal(got[m // 3:first_k, :, 5], ref[m // 3:first_k, :, 5])
    seen = torch.isnan(ref[first_k:]).all(-1) if bad != bad else None
    if seen is not None:
        assert torch.isnan(got[first_k:][seen]).all()


@BITS
def test_strides_of_a_packed_projection_and_an_offset_start(bits):
    """q as a slice of [n, H_q + 2 H_kv, 128]; q_start begins behind rows that belong to nobody."""
    H_q, H_kv, new = 28, 4, [5, 70, 1]
    lens = [50, 300, 1000]
    cache = C.filled(lens, H_q, H_kv, 64, bits)
    big = C.queries(sum(new) + 9, H_q + 2 * H_kv)
    q = big[:, :H_q]
    q_start = torch.tensor([4, 9, 79, 80], dtype=torch.int32, device="cuda")
    chunk = mb.ChunkBatch(cache.kv, q_start, q.shape[0], max_len=70)
    out = torch.full((q.shape[0], H_q, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    call = mb.mage_chunk_attn if bits == 16 else mb.mage_chunk_attn_kv8
    call(cache.kv, chunk, q, 128 ** -0.5, out, chunk.new_workspace(), mask_block=1)
    assert (out[:4] == 7.0).all() and (out[80:] == 7.0).all()
    C.check_attn(cache, q[4:], new, 1, out[4:], None)


def test_token_major_cache():
    """A contiguous cache stored [P][N][H_kv][d]: the row stride is not 128."""
    cache = C.filled([300, 77], 8, 2, 0, 16, head_major=False)
    for new in ([1, 1], [40, 60]):
        q = C.queries(sum(new), 8)
        out, lse = C.run_attn(cache, q, new, 1)
        C.check_attn(cache, q, new, 1, out, lse)


@BITS
@pytest.mark.parametrize("m", [1, 90])
def test_large_logits_move_the_reference(bits, m):
    """Queries 30 times as long: the maximum of a row jumps by tens of binades between tiles.  The tolerance follows the logits:
    |q| |k| d additions of fp32, and the 8-bit query split."""
    cache = C.filled([3000], 8, 2, 64, bits)
    q = C.queries(m, 8, spread=30.0)
    out, lse = C.run_attn(cache, q, [m], 1)
    ref, mag, rl = C.attend(cache, 0, q, 1)
    d_logit = 30 * 5e-4
    assert ((lse - rl).abs() <= d_logit).all()
    assert ((out.double() - ref).abs() <= C.OUT_REL * ref.abs() + (2.0 ** -8 + 2 * d_logit) * mag + C.ABS).all()


@BITS
def test_offsets_beyond_32_bits(bits):
    """Rows more than 2^32 bytes into the pools."""
    H_kv, page = 2, 64
    pages = (2 ** 32 + 2 ** 28) // (H_kv * page * 128)
    lens = [130, 70]
    n = 300 if bits == 16 else 130
    shape = (pages, H_kv, page, 128)
    table = torch.tensor([[pages - 1, 3, pages - 2], [0, pages - 5, -1]], dtype=torch.int32, device="cuda")
    cache = C.Cache(lens, 8, H_kv, page, bits)
    if bits == 16:
        cache.k, cache.v = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache.kv = mb.KVCache(cache.k, cache.v, 8, 1, seq_lens=cache.seq_lens, block_table=table, N_max=130)
    else:
        cache.k, cache.v = (torch.empty(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
        cache.ks, cache.vs = (torch.empty(shape[:3], device="cuda") for _ in range(2))
        cache.kv = mb.Kv8Cache(cache.k, cache.v, cache.ks, cache.vs, 8, seq_lens=cache.seq_lens, block_table=table, N_max=130)
    cache.table = table
    for p, m in enumerate(lens):
        cache.put(p, torch.arange(m), torch.randn(m, H_kv, 128), torch.randn(m, H_kv, 128))
    for new in ([1, 1], [60, 70]):
        q = C.queries(sum(new), 8)
        out, lse = C.run_attn(cache, q, new, 1)
        C.check_attn(cache, q, new, 1, out, lse)


@BITS
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 2, 70]])
def test_bad_pages_and_bad_ranges_are_reported_and_left_out(bits, new):
    lens = [200, 150, 300]
    cache = C.filled(lens, 8, 2, 64, bits)
    q = C.queries(sum(new), 8)
    good, _ = C.run_attn(cache, q, new, 0)
    keep = cache.table[0, 1].item()
    cache.table[0, 1] = 10 ** 6
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, _ = C.run_attn(cache, q, new, 0, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == mb.DEV_BAD_PAGE
    assert torch.equal(out[new[0]:], good[new[0]:])
    # problem 0: as if the keys 64 .. 127 were not there
    k, v = (torch.cat([x[:, :64], x[:, 128:]], 1) for x in _rows_without(cache, keep))
    x = torch.einsum("ihgd,hnd->ihgn", q[:new[0]].double().view(new[0], 2, 4, 128), k) * 128 ** -0.5
    ref = torch.einsum("ihgn,hnd->ihgd", torch.softmax(x, -1), v).reshape(new[0], 8, 128)
    assert ((out[:new[0]].double() - ref).abs() <= 2e-2).all()
    cache.table[0, 1] = keep
    # a problem whose range is no range is skipped, the others are not
    q_start = torch.tensor([0, new[0], new[0] + 10 ** 6, sum(new)], dtype=torch.int32, device="cuda")
    chunk = mb.ChunkBatch(cache.kv, q_start, sum(new), max_len=max(new))
    out = torch.full((sum(new), 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    status.zero_()
    call = mb.mage_chunk_attn if bits == 16 else mb.mage_chunk_attn_kv8
    call(cache.kv, chunk, q, 128 ** -0.5, out, chunk.new_workspace(), mask_block=0, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == mb.DEV_BAD_CHUNK
    assert torch.equal(out[:new[0]], good[:new[0]]) and (out[new[0]:] == 7.0).all()


def _rows_without(cache, keep):
    page = cache.table[0, 1].item()
    cache.table[0, 1] = keep
    rows = cache.rows(0)
    cache.table[0, 1] = page
    return rows


@BITS
@pytest.mark.parametrize("new", [[1] * 6, [50, 1, 0, 200, 3, 9]])
def test_same_bits_every_time_captured_and_on_another_stream(bits, new):
    lens = [5000, 1, 700, 2000, 64, 333]
    lens = [max(a, b) for a, b in zip(lens, new)]
    cache = C.filled(lens, 28, 4, 64, bits)
    q = C.queries(sum(new), 28)
    first, lse = C.run_attn(cache, q, new, 1)
    C.check_attn(cache, q, new, 1, first, lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    with torch.cuda.stream(side):
        other, _ = C.run_attn(cache, q, new, 1, status=status)
    side.synchronize()
    assert torch.equal(other, first)
    # two captured graphs that share one workspace, replayed one after the other, lengths changed between replays
    chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), sum(new), max_len=max(new))
    ws, out = chunk.new_workspace(), torch.empty(2, sum(new), 28, 128, dtype=torch.bfloat16, device="cuda")
    q2 = C.queries(sum(new), 28, seed=9)
    call = mb.mage_chunk_attn if bits == 16 else mb.mage_chunk_attn_kv8
    graphs = []
    for i, x in enumerate((q, q2)):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(cache.kv, chunk, x, 128 ** -0.5, out[i], ws, mask_block=1)
        graphs.append(gr)
    for _ in range(3):
        for gr in graphs:
            gr.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], first)
    C.check_attn(cache, q2, new, 1, out[1], None)
    cache.seq_lens[0] -= 300
    cache.lens[0] -= 300
    graphs[0].replay()
    torch.cuda.synchronize()
    C.check_attn(cache, q, new, 1, out[0], None)


def test_open_chunk_equals_the_exact_pass_on_a_block():
    """A block appended to the cache and attended without a mask is mage_exact_attn of that block."""
    P, H_q, H_kv, N, B = 2, 28, 4, 700, 32
    cache = C.filled([N + B] * P, H_q, H_kv, 0, 16)
    q = C.queries(P * B, H_q)
    out, _ = C.run_attn(cache, q, [B] * P, 0)
    kb, vb = (x[:, :, N:].contiguous() for x in (cache.k, cache.v))
    kv = mb.KVCache(cache.k, cache.v, H_q, B, seq_lens=torch.full((P,), N, dtype=torch.int32, device="cuda"))
    ref = torch.empty(P, H_q, B, 128, dtype=torch.bfloat16, device="cuda")
    mb.mage_exact_attn(kv, q.view(P, B, H_q, 128).transpose(1, 2).contiguous(), kb, vb, 128 ** -0.5, ref, kv.new_workspace())
    got = out.view(P, B, H_q, 128).transpose(1, 2)
    assert ((got.double() - ref.double()).abs() <= 2e-2).all()


@BITS
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [20, 37, 64, 5]])
def test_a_problem_does_not_depend_on_its_neighbours(bits, new):
    """The same call with the other problems' queries, keys and values replaced by NaN gives a problem the same bits."""
    lens = [90, 400, 64, 1000]
    cache = C.filled(lens, 28, 4, 64, bits)
    q = C.queries(sum(new), 28)
    good, lse = C.run_attn(cache, q, new, 1)
    C.check_attn(cache, q, new, 1, good, lse)
    s = C.starts(new)
    for p in (1, 3):
        other = C.filled(lens, 28, 4, 64, bits)
        for x in range(4):
            if x != p:
                nan = torch.full((lens[x], 4, 128), float("nan"))
                other.put(x, torch.arange(lens[x]), nan, nan)
        q2 = torch.full_like(q, float("nan"))
        q2[s[p]:s[p + 1]] = q[s[p]:s[p + 1]]
        out, l2 = C.run_attn(other, q2, new, 1)
        assert torch.equal(out[s[p]:s[p + 1]], good[s[p]:s[p + 1]]) and torch.equal(l2[s[p]:s[p + 1]], lse[s[p]:s[p + 1]])


@BITS
@pytest.mark.parametrize("H_q,H_kv,new", [(8, 2, [3, 1, 2, 0, 4]), (28, 4, [2, 1, 1, 2, 1]), (3, 3, [13, 16, 1, 5, 8]), (16, 1, [1, 0, 1, 1, 1]), (10, 2, [1, 3, 2, 1, 3])])
@pytest.mark.parametrize("mask", [0, 1, 2])
def test_a_few_tokens_each(bits, H_q, H_kv, new, mask):
    """Tiles of eight and of sixteen rows, several tokens in one, lengths around the slices' ends; a token with a NaN value in one."""
    ctx = [130, 15, 700, 3, 5000]
    lens = [c + m for c, m in zip(ctx, new)]
    cache = C.filled(lens, H_q, H_kv, 32, bits)
    q = C.queries(sum(new), H_q)
    out, lse = C.run_attn(cache, q, new, mask)
    C.check_attn(cache, q, new, mask, out, lse)
    v = torch.randn(1, H_kv, 128)
    v[0, :, 9] = float("nan")
    cache.put(0, torch.tensor([lens[0] - 1]), torch.randn(1, H_kv, 128), v)
    out, _ = C.run_attn(cache, q, new, mask)
    ref, mag, _ = C.attend(cache, 0, q[:new[0]], mask)
    got, fin = out[:new[0]].double(), torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fin)
    assert ((got - ref).abs() <= C.OUT_REL * ref.abs() + C.W_REL * mag + C.ABS)[fin].all()


@BITS
@pytest.mark.parametrize("H_q,H_kv,page,mask", [(28, 4, 16, 32), (24, 3, 64, 0), (8, 8, 0, 100)])
def test_many_mixed_chunks(bits, H_q, H_kv, page, mask):
    """Runs of many items of one and of two M-tiles, whole and cut, several times: each call the same bits."""
    g = torch.Generator().manual_seed(11)
    new = (torch.rand(30, generator=g) ** 2 * 500).int().tolist() + [0, 1, 17, 300]
    ctx = (torch.rand(34, generator=g) ** 3 * 4000).int().tolist()
    lens = [c + m for c, m in zip(ctx, new)]
    cache = C.filled(lens, H_q, H_kv, page, bits)
    q = C.queries(sum(new), H_q)
    first, lse = C.run_attn(cache, q, new, mask)
    C.check_attn(cache, q, new, mask, first, lse)
    for _ in range(5):
        out, l = C.run_attn(cache, q, new, mask)
        assert torch.equal(out, first) and torch.equal(l, lse)


@BITS
def test_a_wait_that_runs_out_sets_the_status_and_leaves_the_context_usable(bits):
    """With MAGE_FLAG_TEST_STALL no key tile is requested: the waits give up after about a millisecond and the call returns."""
    new, lens = [150, 40], [700, 40]
    cache = C.filled(lens, 8, 2, 64, bits)
    q = C.queries(sum(new), 8)
    first, _ = C.run_attn(cache, q, new, 1)
    cache.kv.c.flags = mb.FLAG_TEST_STALL
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    C.run_attn(cache, q, new, 1, status=status)
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 5.0
    assert int(status.item()) & mb.DEV_TIMEOUT
    cache.kv.c.flags = 0
    out, lse = C.run_attn(cache, q, new, 1)
    assert torch.equal(out, first)
    C.check_attn(cache, q, new, 1, out, lse)


@BITS
def test_results_at_16_byte_addresses(bits):
    """Outputs that start at an odd multiple of 16 bytes: the same bits, and nothing around them is written."""
    new, lens = [70, 1, 30], [300, 1, 90]
    cache = C.filled(lens, 8, 2, 64, bits)
    q = C.queries(sum(new), 8)
    first, _ = C.run_attn(cache, q, new, 1)
    n = first.numel()
    buf = torch.full((n + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    for at in (8, 24):
        buf.fill_(7.0)
        C.run_attn(cache, q, new, 1, out=buf[at:at + n].view_as(first))
        assert torch.equal(buf[at:at + n].view_as(first), first)
        assert (buf[:at] == 7.0).all() and (buf[at + n:] == 7.0).all()


@pytest.mark.parametrize("big", [1.0, 3.0e4, 1.0e6])
@pytest.mark.parametrize("new,ctx", [([1], 3), ([2], 200), ([20], 2), ([20], 300), ([70], 5), ([70], 700)])
def test_value_rows_of_very_different_scales(new, ctx, big):
    """8-bit cache: a value row that nobody attends, 2^13 to 2^20 times as large as the others, and a row of zeros (whose scale is 1)
    take no precision from the others.  (The tolerance is check_attn's: the large row's weight is below 1e-40.)"""
    cache = C.filled([ctx + new[0]], 8, 2, 64, 8)
    g = torch.Generator().manual_seed(2)
    n = ctx + new[0]
    k, v = 0.1 * torch.randn(n, 2, 128, generator=g), torch.randn(n, 2, 128, generator=g)
    if big == 1.0:
        v = v * 2e-3
    k[1], v[1] = -10.0, big
    v[0] = 0.0
    cache.put(0, torch.arange(n), k, v)
    q = (1.0 + 0.1 * torch.randn(new[0], 8, 128, generator=g)).to(torch.bfloat16).cuda()
    for mask in (0, 1):
        out, lse = C.run_attn(cache, q, new, mask)
        C.check_attn(cache, q, new, mask, out, lse)


@BITS
@pytest.mark.parametrize("new", [1, 150])
def test_starts_that_do_not_ascend_are_reported_and_stay_inside(bits, new):
    lens = [400, 500, 600]
    cache = C.filled(lens, 8, 2, 64, bits)
    n = 3 * new
    q = C.queries(n, 8)
    q_start = torch.tensor([0, 2 * new, new, 3 * new], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    buf = torch.full((n + 20, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    chunk = mb.ChunkBatch(cache.kv, q_start, n, max_len=2 * new)
    call = mb.mage_chunk_attn if bits == 16 else mb.mage_chunk_attn_kv8
    call(cache.kv, chunk, q, 128 ** -0.5, buf[10:10 + n], chunk.new_workspace(), mask_block=1, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == mb.DEV_BAD_CHUNK
    assert (buf[:10] == 7.0).all() and (buf[10 + n:] == 7.0).all()


@BITS
@pytest.mark.parametrize("new", [[4], [36], [5, 40]])
def test_items_of_many_parts(bits, new):
    """Few items over a long cache: tens of partial results each, merged by several blocks; the same bits every time."""
    lens = [30000 - 77 * i for i in range(len(new))]
    cache = C.filled(lens, 28, 4, 16, bits)
    q = C.queries(sum(new), 28)
    first, lse = C.run_attn(cache, q, new, 1)
    C.check_attn(cache, q, new, 1, first, lse)
    for _ in range(3):
        out, l = C.run_attn(cache, q, new, 1)
        assert torch.equal(out, first) and torch.equal(l, lse)


@BITS
@pytest.mark.parametrize("top", [2, 60])
def test_a_padded_batch_captured_once(bits, top):
    """A server's graph: captured at its largest size, replayed with other ranges and lengths, the rows and problems behind the
    last ones untouched."""
    P, H_q, H_kv, n_max = 6, 28, 4, 500
    cache = C.filled([n_max] * P, H_q, H_kv, 64, bits)
    n_tok = P * top
    q = C.queries(n_tok, H_q)
    q_start, out = torch.zeros(P + 1, dtype=torch.int32, device="cuda"), torch.empty(n_tok, H_q, 128, dtype=torch.bfloat16, device="cuda")
    lse, status = torch.empty(n_tok, H_q, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    chunk = mb.ChunkBatch(cache.kv, q_start, n_tok, max_len=top)
    ws = chunk.new_workspace()
    call = mb.mage_chunk_attn if bits == 16 else mb.mage_chunk_attn_kv8
    gr = torch.cuda.CUDAGraph()
    call(cache.kv, chunk, q, 128 ** -0.5, out, ws, lse=lse, dev_status=status)
    torch.cuda.synchronize()
    with torch.cuda.graph(gr):
        call(cache.kv, chunk, q, 128 ** -0.5, out, ws, lse=lse, dev_status=status)
    g = torch.Generator().manual_seed(4)
    for live in (P, 1, 4, 0, 3):
        new = [int(torch.randint(1, top + 1, (1,), generator=g)) if p < live else 0 for p in range(P)]
        lens = [int(torch.randint(m, n_max + 1, (1,), generator=g)) if m else 0 for m in new]
        q_start.copy_(torch.tensor(C.starts(new), dtype=torch.int32))
        cache.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        cache.lens = lens
        out.fill_(7.0)
        lse.fill_(7.0)
        gr.replay()
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        C.check_attn(cache, q, new, 1, out, lse)


@BITS
def test_two_calls_at_once(bits):
    """Two streams, each with its workspace, one with prompts and one with single tokens."""
    lens = [900, 40, 300, 2000]
    cache = C.filled(lens, 28, 4, 64, bits)
    sets = []
    for new in ([200, 40, 1, 90], [1, 1, 1, 1]):
        q = C.queries(sum(new), 28)
        ref, _ = C.run_attn(cache, q, new, 1)
        chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), sum(new), max_len=max(new))
        sets.append((q, ref, chunk, chunk.new_workspace(), torch.empty(20, *ref.shape, dtype=torch.bfloat16, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    call = mb.mage_chunk_attn if bits == 16 else mb.mage_chunk_attn_kv8
    for i in range(20):
        for q, _, chunk, ws, out, stream in sets:
            call(cache.kv, chunk, q, 128 ** -0.5, out[i], ws, stream=stream)
    torch.cuda.synchronize()
    for _, ref, _, _, out, _ in sets:
        assert all(torch.equal(o, ref) for o in out)
