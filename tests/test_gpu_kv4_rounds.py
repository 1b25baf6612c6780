"""The 4-bit cache in a server's round, and the calls around it at sizes whose offsets pass 31 and 32 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import chunk_harness as C
import kv4_harness as K4
from paper_2602_14209_b200 import binding as mb


def test_prompt_in_chunks_then_blocks_over_the_4_bit_cache():
    """Rotated and written in one call, attended -- a prompt in three ragged chunks and two decoded tokens -- then the prefix read back for the exact pass and the
    selection, the selected rows read back for a reuse step."""
    H_q, H_kv, page, P, B, k_sel = 28, 4, 64, 3, 32, 64
    steps = [[100, 33, 7], [40, 0, 64], [1, 200, 1], [1, 1, 1], [1, 1, 1]]
    total = [sum(s[p] for s in steps) for p in range(P)]
    cache = K4.Cache(total, H_q, H_kv, page)
    cache.lens = [0] * P
    cache.seq_lens.zero_()
    rope = mb.Rope((10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda(), axis_of_pair=[0] * 24 + [1] * 20 + [2] * 20)
    for i, new in enumerate(steps):
        n = sum(new)
        qkv = C.queries(n, H_q + 2 * H_kv, seed=20 + i)
        pos = torch.cat([torch.arange(cache.lens[p], cache.lens[p] + m) for p, m in enumerate(new)]).int().cuda().expand(3, n).contiguous()
        cache.lens = [a + b for a, b in zip(cache.lens, new)]
        cache.seq_lens.copy_(torch.tensor(cache.lens, dtype=torch.int32))
        chunk = mb.ChunkBatch(cache.kv, torch.tensor(C.starts(new), dtype=torch.int32, device="cuda"), n, max_len=max(new))
        q, k, v = qkv[:, :H_q], qkv[:, H_q:H_q + H_kv], qkv[:, H_q + H_kv:]
        k_rot = torch.empty(k.shape, dtype=torch.bfloat16, device="cuda")
        mb.mage_rope(rope, pos, q, k, q_out=torch.empty(q.shape, dtype=torch.bfloat16, device="cuda"), k_out=k_rot)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        mb.mage_rope_append_chunk_kv4(cache.kv, chunk, rope, pos, q, k, v, dev_status=status)
        out, lse = torch.full((n, H_q, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((n, H_q), 7.0, device="cuda")
        mb.mage_chunk_attn_kv4(cache.kv, chunk, q, 128 ** -0.5, out, chunk.new_workspace(), mask_block=1, lse=lse, dev_status=status)
        assert int(status.item()) == 0
        C.check_attn(cache, q, new, 1, out, lse)
        s = C.starts(new)
        for p, m in enumerate(new):
            code, u = K4.quantise(k_rot[s[p]:s[p + 1]])
            at = cache.at(p, torch.arange(cache.lens[p] - m, cache.lens[p]))
            assert torch.equal(cache.k[at].cpu(), K4.pack(code)) and torch.equal(cache.ks[at].cpu(), u)
    n_max = max(cache.lens)
    kr, vr = (torch.zeros(P, H_kv, n_max, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv4_read(cache.kv, kr, vr)
    for p in range(P):
        for got, want in zip((kr, vr), cache.rows(p)):
            assert torch.equal(got[p, :, :cache.lens[p]].double(), want)
    kv = mb.KVCache(kr, vr, H_q, B, seq_lens=cache.seq_lens)
    from paper_2602_14209_b200.pipeline import BlockAttention
    ba = BlockAttention(kv, k_sel)
    q, kb, vb = (C.queries(P * B, h, seed=50 + h).view(P, B, h, 128).transpose(1, 2).contiguous() for h in (H_q, H_kv, H_kv))
    ba.exact_select(q, kb, vb)
    ba.select_async()
    ba.join()
    ref = ba.sparse_step(q, kb, vb).clone()
    ks, vs = (torch.zeros(P, H_kv, k_sel, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mb.mage_kv4_read(cache.kv, ks, vs, indices=ba.indices, k_eff=ba.k_eff)
    small = mb.KVCache(ks, vs, H_q, B, seq_lens=ba.k_eff)
    every = torch.arange(k_sel, dtype=torch.int32, device="cuda").expand(P, H_kv, k_sel).contiguous()
    got = torch.empty_like(ref)
    mb.mage_sparse_block_attn(small, q, kb, vb, every, ba.k_eff, k_sel, 128 ** -0.5, got, small.new_workspace(k_sel))
    torch.cuda.synchronize()
    assert torch.equal(got, ref)


def test_contiguous_rows_behind_two_to_the_32_elements():
    """The last problem of a contiguous cache lies behind 5.2e9 elements: written (plainly and rotating), read back, attended."""
    P, H_kv, n_max, n, H_q = 40, 8, 131072, 300, 32
    mk = lambda w: torch.full((P, H_kv, n_max, w), 0xFF, dtype=torch.uint8, device="cuda")
    k, v, ks, vs = mk(64), mk(64), mk(8), mk(8)
    lens = torch.tensor([0] * (P - 1) + [n], dtype=torch.int32, device="cuda")
    kv = mb.Kv4Cache(k, v, ks, vs, H_q, seq_lens=lens)
    start = torch.tensor([0] * P + [n], dtype=torch.int32, device="cuda")
    x = C.queries(n, H_q + 2 * H_kv, seed=3)
    chunk = mb.ChunkBatch(kv, start, n)
    rope = mb.Rope((10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda())
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rotated = torch.empty(n, H_kv, 128, dtype=torch.bfloat16, device="cuda")
    mb.mage_rope(rope, pos, x[:, :H_q], x[:, H_q:H_q + H_kv], q_out=torch.empty(n, H_q, 128, dtype=torch.bfloat16, device="cuda"), k_out=rotated)
    ko, vo = (torch.zeros(P, H_kv, n, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for turn in (False, True):
        keys = rotated if turn else x[:, H_q:H_q + H_kv]
        if turn:
            mb.mage_rope_append_chunk_kv4(kv, chunk, rope, pos, x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:])
        else:
            mb.mage_append_chunk_kv4(kv, chunk, keys, x[:, H_q + H_kv:])
        mb.mage_kv4_read(kv, ko, vo)
        for got, rows in ((ko, keys), (vo, x[:, H_q + H_kv:])):
            c, u = K4.quantise(rows)
            assert torch.equal(got[-1].transpose(0, 1).double(), K4.values(K4.pack(c).cuda(), u.cuda())) and (got[:-1] == 0).all()
        assert all(bool((pool[:-1, :, :n] == 0xFF).all()) and bool((pool[-1, :, n:2 * n] == 0xFF).all()) for pool in (k, v, ks, vs))
    k16 = mb.KVCache(ko, vo, H_q, 1, seq_lens=lens)
    for m in (1, 7, n):                                                    # few rows, one and two groups of them, and many
        q = C.queries(m, H_q, seed=m)
        part = mb.ChunkBatch(kv, torch.tensor([0] * P + [m], dtype=torch.int32, device="cuda"), m)
        out, ref = torch.empty_like(q), torch.empty_like(q)
        mb.mage_chunk_attn_kv4(kv, part, q, 128 ** -0.5, out, part.new_workspace())
        on16 = mb.ChunkBatch(k16, part.q_start, m)
        mb.mage_chunk_attn(k16, on16, q, 128 ** -0.5, ref, on16.new_workspace())
        # each within its own rounding of the same numbers: of the outputs, and of the probabilities over values of at most vo's largest
        assert ((out.double() - ref.double()).abs() <= 2 * (C.OUT_REL * ref.double().abs() + C.W_REL * vo.double().abs().max())).all()


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_rotated_and_written_tokens_behind_two_to_the_31_elements(bits):
    """A token tensor of more than 2^31 elements: as the rotation and the write one after the other."""
    H_q, H_kv, n = 12, 2, 1100000                                          # 16 heads of 128: 2.25e9 elements
    x = torch.randn(4096, H_q + 2 * H_kv, 128, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    x = x.repeat(-(-n // 4096), 1, 1)[:n]
    x[-1000:] = torch.randn(1000, H_q + 2 * H_kv, 128, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rope = mb.Rope((10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda())
    zeros = [torch.zeros(1, H_kv, n, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kinds = {16: lambda: mb.KVCache(zeros[0].clone(), zeros[1].clone(), H_q, 1), 8: lambda: mb.Kv8Cache.like(mb.KVCache(*zeros, H_q, 1)), 4: lambda: mb.Kv4Cache.like(mb.KVCache(*zeros, H_q, 1))}
    one, two = kinds[bits](), kinds[bits]()
    start = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    q, want = (torch.zeros(n, H_q, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k = torch.empty(n, H_kv, 128, dtype=torch.bfloat16, device="cuda")
    form = {16: "", 8: "_kv8", 4: "_kv4"}[bits]
    getattr(mb, "mage_rope_append_chunk" + form)(one, mb.ChunkBatch(one, start, n), rope, pos, x[:, :H_q], x[:, H_q:H_q + H_kv], x[:, H_q + H_kv:], q)
    mb.mage_rope(rope, pos, x[:, :H_q], x[:, H_q:H_q + H_kv], want, k)
    getattr(mb, "mage_append_chunk" + form)(two, mb.ChunkBatch(two, start, n), k, x[:, H_q + H_kv:].contiguous())
    assert torch.equal(q, want)
    names = {16: ("k", "v"), 8: ("k8", "v8", "k_scale", "v_scale"), 4: ("k4", "v4", "k_scale", "v_scale")}[bits]
    for name in names:
        assert torch.equal(getattr(one, name), getattr(two, name))
    assert bool((q[-1000:] != 0).any()) and bool((getattr(one, names[0])[0, :, -1000:] != 0).any())
