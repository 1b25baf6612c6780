"""Plain 64-bit implementations of the calls on packed chunks, and builders of caches whose unused rows hold NaN patterns.

Tolerance of an attention output, element by element, from the roundings it has by construction: the output's own (half a
bf16 step, 2^-8 relative), and the probabilities' (2^-8 relative each, so at most 2^-8 * sum_j w_j |v_j|).  Logits: 128 fp32
additions and, for 8-bit keys, the query split's 2^-17 of the row's largest element per product; for unit-normal inputs
their worst case is below 5e-4 absolute, i.e. 1e-3 relative on a weight ratio.  lse is off by at most the logits' error.
"""
import torch

from paper_2602_14209_b200 import binding as mb

D = 128
OUT_REL, W_REL, ABS, LSE_ABS = 2.0 ** -8, 2.0 ** -8 + 1e-3, 1e-6, 5e-4
NAN16, NAN8 = 0x7FC1, 0x7F


def quantise(x):
    """[..., 128] -> (codes as float8, scale): the definition, in single precision on the CPU."""
    x = x.float().cpu()
    amax = x.abs().amax(-1)
    s = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
    code = (x / s[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    odd = ~torch.isfinite(x).all(-1)
    s[odd] = float("nan")
    code.view(torch.uint8)[odd] = 0
    return code, s


class Cache:
    """A 16- or 8-bit cache, contiguous (page 0) or paged, all rows NaN until ``put`` writes them."""

    def __init__(self, lens, H_q, H_kv, page, bits, n_max=None, seed=0, head_major=True):
        self.lens, self.H_q, self.H_kv, self.page, self.bits, P = list(lens), H_q, H_kv, page, bits, len(lens)
        self.n_max = max(max(lens), 1) if n_max is None else n_max
        g = torch.Generator().manual_seed(seed)
        self.table = None
        if page:
            per = [-(-n // page) for n in lens]
            ids = torch.randperm(sum(per) + 3, generator=g).int()
            table = torch.full((P, -(-self.n_max // page)), -1, dtype=torch.int32)
            at = 0
            for p, m in enumerate(per):
                table[p, :m] = ids[at:at + m]
                at += m
            self.table, shape = table.cuda(), (sum(per) + 3, H_kv, page, D)
        else:
            shape = (P, H_kv, self.n_max, D)
        if bits == 16:
            mk = lambda: torch.full(shape if head_major or page else (P, self.n_max, H_kv, D), NAN16, dtype=torch.int16, device="cuda").view(torch.bfloat16)
            self.k, self.v = mk(), mk()
            if not head_major and not page:
                self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        else:
            self.k, self.v = (torch.full(shape, NAN8, dtype=torch.uint8, device="cuda") for _ in range(2))
            self.ks, self.vs = (torch.full(shape[:3], float("nan"), device="cuda") for _ in range(2))
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        N = self.n_max
        if bits == 16:
            self.kv = mb.KVCache(self.k, self.v, H_q, 1, seq_lens=self.seq_lens, block_table=self.table, N_max=N)
        else:
            self.kv = mb.Kv8Cache(self.k, self.v, self.ks, self.vs, H_q, seq_lens=self.seq_lens, block_table=self.table, N_max=N if page else None)

    def at(self, p, j):
        """Index of rows j (tensor) of problem p in the pools: x[index] is [len(j), H_kv, ...]."""
        j = j.cuda()
        return (self.table[p].long()[j // self.page], slice(None), j % self.page) if self.page else (p, slice(None), j)

    def put(self, p, j, k, v):
        """Rows j of problem p from k, v [len(j), H_kv, 128]."""
        i = self.at(p, j)
        if not self.page:
            k, v = k.transpose(0, 1), v.transpose(0, 1)          # (one integer index: the sliced dimension comes first)
        if self.bits == 16:
            self.k[i], self.v[i] = k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16).cuda()
        else:
            for x, pool, sc in ((k, self.k, self.ks), (v, self.v, self.vs)):
                c, s = quantise(x)
                pool[i], sc[i] = c.view(torch.uint8).cuda(), s.cuda()

    def rows(self, p, n=None):
        """(k, v) of the first n rows as they stand, [H_kv, n, 128] float64."""
        n = self.lens[p] if n is None else n
        i = self.at(p, torch.arange(n))
        out = []
        for pool, sc in ((self.k, None), (self.v, None)) if self.bits == 16 else ((self.k, self.ks), (self.v, self.vs)):
            x = pool[i]
            x = x.double() if sc is None else x.view(torch.float8_e4m3fn).double() * sc[i].double()[..., None]
            out.append(x.transpose(0, 1) if self.page else x)
        return out


def filled(lens, H_q, H_kv, page, bits, seed=0, **kw):
    c = Cache(lens, H_q, H_kv, page, bits, seed=seed, **kw)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    for p, n in enumerate(lens):
        if n:
            k, v = (torch.randn(n, H_kv, D, generator=g, device="cuda") for _ in range(2))
            c.put(p, torch.arange(n), k, v)
    return c


def starts(new):
    s = [0]
    for m in new:
        s.append(s[-1] + m)
    return s


def visible(t, n, b):
    return 0 if t < 0 else n if b == 0 else min(n, (t // b + 1) * b)


def attend(cache, p, q, mask, scale=D ** -0.5):
    """Problem p's new tokens q [m, H_q, 128] by the definition in 64 bits: (out, sum_j w_j |v_j|, lse), keys that a row does not
    see taken out of the arrays before anything is computed from them."""
    m, G, n = q.shape[0], cache.H_q // cache.H_kv, cache.lens[p]
    k, v = cache.rows(p)
    out, mag = (torch.zeros(m, cache.H_q, D, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((m, cache.H_q), float("-inf"), dtype=torch.float64, device="cuda")
    ends = [visible(n - m + i, n, mask) for i in range(m)]
    for e in sorted(set(ends)):
        if e == 0:
            continue
        i = torch.tensor([x for x in range(m) if ends[x] == e], device="cuda")
        x = torch.einsum("ihgd,hnd->ihgn", q[i].double().view(len(i), cache.H_kv, G, D), k[:, :e]) * scale
        w = torch.softmax(x, -1)
        out[i] = torch.einsum("ihgn,hnd->ihgd", w, v[:, :e]).reshape(len(i), -1, D)
        mag[i] = torch.einsum("ihgn,hnd->ihgd", w, v[:, :e].abs()).reshape(len(i), -1, D)
        lse[i] = torch.logsumexp(x, -1).reshape(len(i), -1)
    return out, mag, lse


def run_attn(cache, q, new, mask, lse=True, pad=0, max_len=None, stream=None, status=None, scale=D ** -0.5, workspace=None, out=None):
    s = starts(new)
    q_start = torch.tensor(s, dtype=torch.int32, device="cuda")
    n = q.shape[0]
    chunk = mb.ChunkBatch(cache.kv, q_start, n, max_len=max(new) if max_len is None else max_len)
    out = torch.full((n, cache.H_q, D), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    l = torch.full((n, cache.H_q), 7.0, device="cuda") if lse else None
    own = status is None
    status = torch.zeros(1, dtype=torch.int32, device="cuda") if own else status
    ws = chunk.new_workspace().fill_(0xFF) if workspace is None else workspace
    call = mb.mage_chunk_attn if cache.bits == 16 else mb.mage_chunk_attn_kv8
    call(cache.kv, chunk, q, scale, out, ws, mask_block=mask, lse=l, dev_status=status, stream=stream)
    if own:
        torch.cuda.synchronize()
        assert int(status.item()) == 0
    return out, l


def check_attn(cache, q, new, mask, out, lse, scale=D ** -0.5, problems=None):
    s = starts(new)
    for p, m in enumerate(new):
        if m == 0 or (problems is not None and p not in problems):
            continue
        ref, mag, rl = attend(cache, p, q[s[p]:s[p + 1]], mask, scale)
        got = out[s[p]:s[p + 1]].double()
        same = torch.isnan(ref)
        assert torch.equal(torch.isnan(got), same), f"problem {p}: NaN in other places"
        fin = torch.isfinite(ref)
        assert torch.equal(got[~fin & ~same], ref[~fin & ~same])
        err = (got - ref).abs() - (OUT_REL * ref.abs() + W_REL * mag + ABS)
        assert (err[fin] <= 0).all(), (p, float((got - ref).abs()[fin].max()))
        if lse is not None:
            gl = lse[s[p]:s[p + 1]].double()
            dead = rl == float("-inf")
            assert torch.equal(gl == float("-inf"), dead) and torch.equal(torch.isnan(gl), torch.isnan(rl))
            ok = torch.isfinite(rl)
            assert ((gl - rl).abs()[ok] <= LSE_ABS).all(), (p, float((gl - rl).abs()[ok].max()))
    assert (out[s[-1]:] == 7.0).all()
    if lse is not None:
        assert (lse[s[-1]:] == 7.0).all()


def queries(n, H_q, seed=3, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, H_q, D, generator=g, device="cuda") * spread).to(torch.bfloat16)
