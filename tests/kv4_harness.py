"""The 4-bit cache by its definition, in 64 bits on the CPU, and caches of it whose unused rows hold anything.

Attention over it has the roundings of the 16-bit cache, since every value of the format is a bf16 number: the tolerances of
``chunk_harness`` for 16 bits hold as they are (probabilities rounded to bf16, the output's own rounding, fp32 sums of 128 products).
"""
import torch

import chunk_harness as C
from paper_2602_14209_b200 import binding as mb

D = 128
SCALES = torch.tensor([2.0 ** (i // 8 - 17) * (1 + i % 8 / 8) for i in range(248)], dtype=torch.float64)


def quantise(x):
    """[..., 128] bf16 -> (codes [..., 128] as whole numbers, scale bytes [..., 8]): the nearest scale to amax / 7 (halves up), the nearest
    code to x / s (halves toward zero), 7 at most."""
    g = x.double().cpu().reshape(x.shape[:-1] + (8, 16))
    odd = ~torch.isfinite(x.double().cpu()).all(-1)
    g = torch.where(odd[..., None, None], 0.0, g)
    u = torch.searchsorted((SCALES[1:] + SCALES[:-1]) / 2, g.abs().amax(-1) / 7, right=True)
    t = g / SCALES[u][..., None]
    c = (torch.sign(t) * torch.ceil(t.abs() - 0.5)).clamp(-7, 7).long().reshape(x.shape)
    u[odd] = 255
    return c, u.to(torch.uint8)


def pack(c):
    w = (c + 8).reshape(c.shape[:-1] + (16, 8))
    word = sum(w[..., e] << (4 * (e // 2) + 16 * (e % 2)) for e in range(8))
    return torch.stack([(word >> s) & 255 for s in (0, 8, 16, 24)], -1).to(torch.uint8).reshape(c.shape[:-1] + (64,))


def values(codes, u):
    """What packed codes and scale bytes stand for, in 64 bits, on their device."""
    b = codes.reshape(codes.shape[:-1] + (16, 4)).long()
    word = b[..., 0] | b[..., 1] << 8 | b[..., 2] << 16 | b[..., 3] << 24
    c = torch.stack([(word >> (4 * (e // 2) + 16 * (e % 2))) & 15 for e in range(8)], -1).reshape(codes.shape[:-1] + (D,)) - 8
    s = torch.cat([SCALES, torch.full((8,), float("nan"), dtype=torch.float64)]).to(u.device)[u.long()]
    return c.double() * s.repeat_interleave(16, -1)


class Cache(C.Cache):
    """A 4-bit cache, contiguous (page 0) or paged, all rows NaN until ``put`` writes them."""

    def __init__(self, lens, H_q, H_kv, page, n_max=None, seed=0, token_major=False):
        super().__init__(lens, H_q, H_kv, page, 8, n_max=n_max, seed=seed)
        self.bits, rows = 4, tuple(self.ks.shape)
        if token_major and not page:
            mk = lambda: torch.full((rows[0], rows[2], rows[1], 64), 0xFF, dtype=torch.uint8, device="cuda").transpose(1, 2)
        else:
            mk = lambda: torch.full(rows + (64,), 0xFF, dtype=torch.uint8, device="cuda")
        self.k, self.v = mk(), mk()
        self.ks, self.vs = (torch.full(rows + (8,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.kv = mb.Kv4Cache(self.k, self.v, self.ks, self.vs, H_q, seq_lens=self.seq_lens, block_table=self.table, N_max=self.n_max if page else None)

    def put(self, p, j, k, v):
        i = self.at(p, j)
        if not self.page:
            k, v = k.transpose(0, 1), v.transpose(0, 1)
        for x, pool, sc in ((k, self.k, self.ks), (v, self.v, self.vs)):
            c, u = quantise(x.to(torch.bfloat16))
            pool[i], sc[i] = pack(c).cuda(), u.cuda()

    def rows(self, p, n=None):
        n = self.lens[p] if n is None else n
        i = self.at(p, torch.arange(n))
        return [(x.transpose(0, 1) if self.page else x) for x in (values(self.k[i], self.ks[i]), values(self.v[i], self.vs[i]))]


def filled(lens, H_q, H_kv, page, seed=0, **kw):
    c = Cache(lens, H_q, H_kv, page, seed=seed, **kw)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    for p, n in enumerate(lens):
        if n:
            k, v = (torch.randn(n, H_kv, D, generator=g, device="cuda") for _ in range(2))
            c.put(p, torch.arange(n), k, v)
    return c


def run_attn(cache, q, new, mask, lse=True, max_len=None, stream=None, status=None, scale=D ** -0.5, workspace=None, out=None):
    q_start = torch.tensor(C.starts(new), dtype=torch.int32, device="cuda")
    n = q.shape[0]
    chunk = mb.ChunkBatch(cache.kv, q_start, n, max_len=max(new) if max_len is None else max_len)
    out = torch.full((n, cache.H_q, D), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    l = torch.full((n, cache.H_q), 7.0, device="cuda") if lse else None
    own = status is None
    status = torch.zeros(1, dtype=torch.int32, device="cuda") if own else status
    ws = chunk.new_workspace().fill_(0xFF) if workspace is None else workspace
    mb.mage_chunk_attn_kv4(cache.kv, chunk, q, scale, out, ws, mask_block=mask, lse=l, dev_status=status, stream=stream)
    if own:
        torch.cuda.synchronize()
        assert int(status.item()) == 0
    return out, l
