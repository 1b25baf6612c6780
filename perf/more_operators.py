"""Cases of the 4-bit cache (written, read back, attended) and of cache writes that rotate the positions on the way.

``run`` computes a case in plain torch (32 bits, rounded once at the end) or, with ``own`` set, by the library's calls.
Both take the same state: packed projections of the new tokens, a paged or contiguous cache, page table, lengths.

4-bit row of 128: eight groups of 16 elements, each with a scale s = 2^(E - 17) (1 + M / 8) in one byte u = 8 E + M (248 and up: not a
number), the nearest to amax / 7 (halves up); a code c = -7 .. 7 is the nearest integer to x / s (halves toward zero), stored as c + 8;
of eight elements in a 32-bit word element 2 i has bits 4 i .. 4 i + 3 and element 2 i + 1 bits 16 + 4 i .. 19 + 4 i.
"""
import math
import random

import torch

own = False

D = 128                                      # head dimension
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoding step of a serving batch: each sequence's q and k are rotated, k and v written to the 16-bit cache; latency counts
        dict(name="write16_step", op="write", bits=16, rope=True, seqs=48, mix=3, ctx_lo=1, ctx_hi=1000, new_lo=1, new_hi=1, hq=28, hkv=4, page=64, axes=3, rot=128,
             halves=True),
        # prompts of 16 requests with images: rotated and written in one call, the bandwidth-bound end
        dict(name="write16_prompt", op="write", bits=16, rope=True, seqs=16, mix=4, ctx_lo=0, ctx_hi=500, new_lo=300, new_hi=2048, hq=32, hkv=8, page=64, axes=3, rot=128,
             halves=True),
        # the same requests on a server that keeps 8 bits, the new rows read back for the first block
        dict(name="write8_prompt", op="write", bits=8, rope=True, seqs=16, mix=4, ctx_lo=0, ctx_hi=500, new_lo=300, new_hi=2048, hq=32, hkv=8, page=64, axes=3, rot=128,
             halves=True),
        # a finished block of 32 tokens of each of 9 sequences: rotated, written in 4 bits, and its rows read back for the next block's first step
        dict(name="write4_block", op="write", bits=4, rope=True, seqs=9, mix=5, ctx_lo=1, ctx_hi=1000, new_lo=32, new_hi=32, hq=28, hkv=4, page=64, axes=3, rot=128,
             halves=True),
        # prompts that are rotated already, written in 4 bits and read back for the first block
        dict(name="write4_prompt", op="write", bits=4, rope=False, seqs=16, mix=4, ctx_lo=0, ctx_hi=500, new_lo=300, new_hi=2048, hq=32, hkv=8, page=64, axes=1, rot=128,
             halves=True),
        # the rows that a block selected, read back once per block for its reuse steps (28 layers, k = 512)
        dict(name="read4_selected", op="read4", seqs=28, mix=5, ctx_lo=4096, ctx_hi=8192, hq=28, hkv=4, page=64, k=512),
        # whole prefixes read back into a 16-bit cache
        dict(name="read4_prefix", op="read4", seqs=2, mix=6, ctx_lo=32000, ctx_hi=32768, hq=32, hkv=8, page=0, k=0),
        # the smallest call: one token of one sequence over a short cache
        dict(name="attn4_step_short", op="attn4", seqs=1, mix=7, ctx_lo=2047, ctx_hi=2047, new_lo=1, new_hi=1, hq=8, hkv=2, page=64, mask=1),
        # a decoding step of 32 sequences of one token to 128K
        dict(name="attn4_step_ragged", op="attn4", seqs=32, mix=10, ctx_lo=0, ctx_hi=131071, new_lo=1, new_hi=1, hq=28, hkv=4, page=64, mask=1),
        # a prompt chunk with a block-causal mask (blocks of 32), odd length
        dict(name="attn4_prompt", op="attn4", seqs=1, mix=11, ctx_lo=16384, ctx_hi=16384, new_lo=2001, new_hi=2001, hq=32, hkv=8, page=64, mask=32),
        # one chunk of a long prompt: 4096 new tokens behind 32K earlier ones, causal, contiguous cache
        dict(name="attn4_prompt_long", op="attn4", seqs=1, mix=9, ctx_lo=32768, ctx_hi=32768, new_lo=4096, new_hi=4096, hq=28, hkv=4, page=0, mask=1),
        # chunks of one to 700 tokens of 24 sequences in one call, small pages
        dict(name="attn4_mixed", op="attn4", seqs=24, mix=12, ctx_lo=0, ctx_hi=16384, new_lo=1, new_hi=700, hq=28, hkv=4, page=16, mask=32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 2)))) - 1))


def draw(rng):
    hq, hkv = rng.choice([(28, 4), (32, 8), (8, 2), (16, 16), (5, 1), (24, 3)])
    page = rng.choice([0, 16, 32, 64, 128])
    mix = rng.randrange(1 << 20)
    op = rng.choice(["write", "write", "read4", "attn4", "attn4", "attn4"])
    if op == "write":
        bits = rng.choice([16, 8, 4, 4])
        new_hi = _log_int(rng, 1, 2048)
        return dict(op=op, bits=bits, rope=bits != 4 or rng.random() < 0.6, seqs=_log_int(rng, 1, max(1, min(64, 16384 // new_hi))), mix=mix, ctx_lo=0,
                    ctx_hi=_log_int(rng, 1, 1000), new_lo=1, new_hi=new_hi, hq=hq, hkv=hkv, page=page, axes=rng.choice([1, 2, 3]), rot=rng.choice([128, 128, 64, 96, 80]),
                    halves=rng.random() < 0.7)
    if op == "read4":
        hi = _log_int(rng, 1, 16384)
        return dict(op=op, seqs=_log_int(rng, 1, max(1, min(28, 32768 // hi))), mix=mix, ctx_lo=1, ctx_hi=hi, hq=hq, hkv=hkv, page=page,
                    k=rng.choice([0, _log_int(rng, 1, 1024)]))
    mask = rng.choice([1, 1, 0, 32, 7])
    if rng.random() < 0.5:                   # a decoding step, or a few tokens each
        hi = _log_int(rng, 1, 131072)
        return dict(op=op, seqs=_log_int(rng, 1, max(1, min(64, 524288 // hi))), mix=mix, ctx_lo=0, ctx_hi=hi, new_lo=1, new_hi=rng.choice([1, 1, 4, 9]), hq=hq, hkv=hkv,
                    page=page, mask=mask)
    new_hi = _log_int(rng, 2, 2048)          # chunks of prompts
    return dict(op=op, seqs=_log_int(rng, 1, max(1, min(16, 4096 // new_hi))), mix=mix, ctx_lo=0, ctx_hi=_log_int(rng, 1, 16384), new_lo=1, new_hi=new_hi, hq=hq, hkv=hkv,
                page=page, mask=mask)


def _lengths(case):
    """Earlier and new tokens of each sequence, from the case alone."""
    rng = random.Random(case["mix"])
    ctx = [_log_int(rng, case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    new = [_log_int(rng, case["new_lo"], case["new_hi"]) if "new_hi" in case else 0 for _ in range(case["seqs"])]
    return ctx, new


def _visible(case, n, t):
    """Keys that the query at position t of a sequence of n tokens sees."""
    b = case["mask"]
    return n if b == 0 else min(n, (t // b + 1) * b)


ROW4 = D // 2 + 8                            # bytes of a 4-bit row


def work(case):
    hq, hkv = case["hq"], case["hkv"]
    ctx, new = _lengths(case)
    if case["op"] == "write":
        n, bits = sum(new), case["bits"]
        nbytes = n * hkv * 2 * (2 * D + {16: 2 * D, 8: D + 4, 4: ROW4}[bits])
        flops = n * hkv * 2 * D * (0 if bits == 16 else 2)
        if case["rope"]:
            nbytes += n * (hq * 4 * D + 4 * case["axes"]) + 2 * case["rot"]
            flops += n * (hq + hkv) * case["rot"] * 3
        if bits < 16:                        # (the new rows are read where they were just written)
            nbytes += n * hkv * 2 * (2 * D + {8: D + 4, 4: ROW4}[bits])
        return {"bytes": nbytes, "flops": flops}
    if case["op"] == "read4":
        rows = sum(min(n, case["k"]) if case["k"] else n for n in ctx) * hkv
        return {"bytes": rows * 2 * (ROW4 + 2 * D) + (4 * rows if case["k"] else 0), "flops": rows * 2 * D}
    nbytes, pairs = sum(new) * hq * (2 * D * 2 + 4), 0
    for c, m in zip(ctx, new):
        nbytes += (c + m) * hkv * 2 * ROW4
        pairs += sum(_visible(case, c + m, c + i) for i in range(m))
    return {"bytes": nbytes, "flops": 4 * D * hq * pairs}


# ------------------------------------------------------------------------------------------------------- the state
def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + sum(ord(c) * 131 ** i for i, c in enumerate(what))) & 0x7FFFFFFFFFFF)
    return g


def _positions(case, ctx, new, seed):
    """[axes][tokens] int32: text advances all axes together, an image gives its rows and columns and stands still in time."""
    rng, rows = random.Random(seed), [[] for _ in range(case["axes"])]
    for c, m in zip(ctx, new):
        at, left = c * rng.choice([1, 1, 40]), m           # (some sequences are far into a long context)
        while left:
            n = min(left, rng.randrange(1, 400))
            w = rng.randrange(2, 30) if case["axes"] > 1 and rng.random() < 0.5 else 0
            for a, r in enumerate(rows):
                r += [at + (0 if a == 0 else i // w if a == 1 else i % w) if w else at + i for i in range(n)]
            at, left = at + n, left - n
    return torch.tensor(rows, dtype=torch.int32, device="cuda")


def _axis_of_pair(case):
    """Which axis turns pair i: contiguous sections, the first axis taking what does not divide."""
    pairs, axes = case["rot"] // 2, case["axes"]
    per = pairs // axes
    first = pairs - per * (axes - 1)
    return [0] * first + [a for a in range(1, axes) for _ in range(per)]


def _code8(x):
    """Rows of [..., 128] in 32 bits -> (e4m3 codes, scale of each row): scale = amax / 448, code = x / scale to nearest even."""
    amax = x.abs().amax(-1)
    s = torch.where(amax > 0, amax / E4M3_MAX, torch.ones_like(amax))
    return (x / s[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), s


def _code4(x):
    """Rows of [..., 128] in 32 bits -> (packed codes [..., 64], scale bytes [..., 8])."""
    g = x.reshape(x.shape[:-1] + (8, 16))
    m, e = torch.frexp(g.abs().amax(-1) / 7)                # m in [1/2, 1): sixteenths are the grid of scales
    s = torch.ldexp(torch.floor(m * 16 + 0.5) / 16, e).clamp(2.0 ** -17, 15360.0)
    m, e = torch.frexp(s)
    u = (e + 16) * 8 + (m * 16 - 8).to(torch.int32)
    t = g / s[..., None]
    c = (torch.sign(t) * torch.ceil(t.abs() - 0.5)).clamp(-7, 7).to(torch.int32) + 8
    c = c.view(x.shape[:-1] + (16, 8))
    b = torch.stack([c[..., 0] | c[..., 2] << 4, c[..., 4] | c[..., 6] << 4, c[..., 1] | c[..., 3] << 4, c[..., 5] | c[..., 7] << 4], -1)
    return b.to(torch.uint8).view(x.shape[:-1] + (64,)), u.to(torch.uint8)


def _value4(codes, u):
    """Packed codes [..., 64] and scale bytes [..., 8] -> rows [..., 128] in 32 bits (exact)."""
    b = codes.view(codes.shape[:-1] + (16, 4)).to(torch.int32)
    lo, hi = b & 15, b >> 4
    c = torch.stack([lo[..., 0], lo[..., 2], hi[..., 0], hi[..., 2], lo[..., 1], lo[..., 3], hi[..., 1], hi[..., 3]], -1).view(u.shape + (16,)) - 8
    u = u.to(torch.int32)
    s = torch.ldexp(1 + (u & 7).float() / 8, (u >> 3) - 17)
    return (c * s[..., None]).view(codes.shape[:-1] + (D,))


def _cache(case, lens, seed, bits, empty=False):
    """Cache of the case: paged pools with a shuffled page table, or one contiguous tensor.  Values as they meet in earnest: unit
    normal with a common direction in one key of 64."""
    hkv, page, seqs = case["hkv"], case["page"], case["seqs"]
    n_max = max(max(lens), 1)
    s = {"n_max": n_max, "seq_lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "table": None}
    if page:
        per = [-(-n // page) for n in lens]
        order = list(range(sum(per) + 2))
        random.Random(seed).shuffle(order)
        table = [[-1] * max(max(per), 1) for _ in lens]
        at = 0
        for p, m in enumerate(per):
            table[p][:m] = order[at:at + m]
            at += m
        s["table"] = torch.tensor(table, dtype=torch.int32, device="cuda")
        shape = (len(order), hkv, page)
    else:
        shape = (seqs, hkv, n_max)
    u = torch.randn(hkv, D, generator=_gen(seed, "u"), device="cuda")
    s["u"] = u / u.norm(dim=-1, keepdim=True)
    width, kind = {16: (D, torch.bfloat16), 8: (D, torch.uint8), 4: (D // 2, torch.uint8)}[bits]
    for what in ("k", "v"):
        pool = torch.zeros(shape + (width,), dtype=kind, device="cuda")
        scale = {16: None, 8: torch.zeros(shape, device="cuda"), 4: torch.zeros(shape + (8,), dtype=torch.uint8, device="cuda")}[bits]
        g = _gen(seed, what)
        if not empty:                        # (4 bits)
            step = max(1, (1 << 26) // (hkv * shape[2] * D))
            for a in range(0, shape[0], step):
                x = torch.randn((min(step, shape[0] - a),) + shape[1:] + (D,), generator=g, device="cuda")
                if what == "k":
                    x[:, :, ::64] += 6.0 * s["u"][:, None, :]
                pool[a:a + step], scale[a:a + step] = _code4(x.to(torch.bfloat16).float())
        s[what], s[what + "s"] = pool, scale
    return s


def prepare(case, seed):
    hq, hkv, op = case["hq"], case["hkv"], case["op"]
    bits = case.get("bits", 4)
    ctx, new = _lengths(case)
    lens = [c + m for c, m in zip(ctx, new)]
    s = _cache(case, lens, seed, bits, empty=op == "write")
    g = _gen(seed, "new")
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    s.update(case=case, ctx=ctx, new=new, lens=lens, starts=starts, q_start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    if op != "read4":
        x = torch.randn(starts[-1], hq + 2 * hkv, D, generator=g, device="cuda")
        x[:, :hq] += 2.0 * s["u"].repeat_interleave(hq // hkv, 0)
        s["qkv"] = x.to(torch.bfloat16)
    if op == "write":                        # token i of the packed batch: its sequence and its position there
        s["seq_of"] = torch.tensor([p for p, m in enumerate(new) for _ in range(m)], device="cuda")
        s["pos_of"] = torch.tensor([c + i for c, m in zip(ctx, new) for i in range(m)], device="cuda")
        s["row_of"] = torch.tensor([i for m in new for i in range(m)], device="cuda")
        s["pos"] = _positions(case, ctx, new, seed)
        pairs = case["rot"] // 2
        s["inv_freq"] = (1e6 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)).float().cuda()
        s["axis"] = torch.tensor(_axis_of_pair(case), device="cuda")
        s["q_out"] = torch.empty(starts[-1], hq, D, dtype=torch.bfloat16, device="cuda")
    rows = max(new) if op == "write" else case["k"] or s["n_max"] if op == "read4" else 0
    if rows and bits < 16:                   # rows to read back: the new ones, the selected ones (ascending), or all; -1 behind a sequence's last
        s["k_out"] = torch.zeros(case["seqs"], hkv, rows, D, dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"])
        if op == "write" or case["k"]:
            pick = torch.full((case["seqs"], hkv, rows), -1, dtype=torch.int32, device="cuda")
            for p, n in enumerate(lens):
                m = new[p] if op == "write" else min(n, case["k"])
                pick[p, :, :m] = torch.arange(n - m, n, device="cuda").int() if op == "write" else torch.rand(hkv, n, generator=g, device="cuda").topk(m, -1).indices.sort(-1).values.int()
            s["pick"] = pick
            s["k_eff"] = torch.tensor(new if op == "write" else [min(n, case["k"]) for n in lens], dtype=torch.int32, device="cuda")
    if op == "attn4":
        s["out"] = torch.empty(starts[-1], hq, D, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty(starts[-1], hq, device="cuda")
    if own:
        from paper_2602_14209_b200 import binding as mb
        if bits == 16:
            s["kv"] = mb.KVCache(s["k"], s["v"], hq, 1, seq_lens=s["seq_lens"], block_table=s["table"], N_max=s["n_max"])
        else:
            s["kv"] = (mb.Kv8Cache if bits == 8 else mb.Kv4Cache)(s["k"], s["v"], s["ks"], s["vs"], hq, seq_lens=s["seq_lens"], block_table=s["table"], N_max=s["n_max"])
        if op != "read4":
            s["chunk"] = mb.ChunkBatch(s["kv"], s["q_start"], n_tokens=starts[-1], max_len=max(new))
        if op == "write":
            s["rope"] = mb.Rope(s["inv_freq"], axis_of_pair=_axis_of_pair(case), rot_dim=case["rot"], halves=case["halves"])
        if op == "attn4":
            s["workspace"] = s["chunk"].new_workspace()
    return s


# ---------------------------------------------------------------------------------------------------- the plain form
def _rotated(s):
    """Queries and keys of the new tokens, rotated, in bf16."""
    case = s["case"]
    rot, n_heads = case["rot"], case["hq"] + case["hkv"]
    angle = s["pos"].double()[s["axis"]].T * s["inv_freq"].double()          # [tokens][pairs]; far positions need 64 bits
    c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = s["qkv"][:, :n_heads].float()
    y = x.clone()
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if case["halves"] else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., lo] = x[..., lo] * c - x[..., hi] * n
    y[..., hi] = x[..., hi] * c + x[..., lo] * n
    return y.to(torch.bfloat16)


def _picked(s):
    """The rows to read back, [sequences][heads][rows][128] in 32 bits twice (zeros behind a sequence's last)."""
    case, out = s["case"], []
    seqs, hkv, rows = s["k_out"].shape[:3]
    j = s["pick"].long() if "pick" in s else torch.arange(rows, device="cuda").expand(seqs, hkv, rows)
    ok = (j >= 0) & (j < s["seq_lens"][:, None, None])
    j = j.clamp(min=0)
    p, h = torch.arange(seqs, device="cuda")[:, None, None], torch.arange(hkv, device="cuda")[None, :, None]
    if case["page"]:
        j = j.clamp(max=s["table"].shape[1] * case["page"] - 1)
        where = (s["table"][p, j // case["page"]].clamp(min=0).long(), h, j % case["page"])
    else:
        where = (p, h, j)
    for what in ("k", "v"):
        codes, scales = s[what][where], s[what + "s"][where]
        x = _value4(codes, scales) if scales.dtype == torch.uint8 else codes.view(torch.float8_e4m3fn).float() * scales[..., None]
        out.append(torch.where(ok[..., None], x, 0.0))
    return out


def _write(s):
    case = s["case"]
    hq, hkv, page, bits = case["hq"], case["hkv"], case["page"], case["bits"]
    out = {}
    qk = s["qkv"][:, :hq + hkv]
    if case["rope"]:
        qk = _rotated(s)
        s["q_out"].copy_(qk[:, :hq])
        out["q"] = s["q_out"]
    p, t = s["seq_of"], s["pos_of"]
    where = (s["table"][p, t // page].long(), slice(None), t % page) if page else (p, slice(None), t)
    for what, new in (("k", qk[:, hq:]), ("v", s["qkv"][:, hq + hkv:])):
        if bits == 16:
            s[what][where] = new
        else:
            codes, scales = (_code8 if bits == 8 else _code4)(new.float())
            s[what][where] = codes.view(torch.uint8)
            s[what + "s"][where] = scales
    if bits == 16:
        return {**out, "k": s["k"], "v": s["v"]}
    return {**out, **_read4(s)}


def _read4(s):
    k, v = _picked(s)
    s["k_out"].copy_(k)
    s["v_out"].copy_(v)
    return {"k": s["k_out"], "v": s["v_out"]}


def _rows(s, p):
    """The keys and values of sequence p as [hkv][n][128] in 32 bits."""
    n, page, out = s["lens"][p], s["case"]["page"], []
    for what in ("k", "v"):
        if page:
            ids = s["table"][p, :-(-n // page)].long()
            x = _value4(s[what][ids], s[what + "s"][ids]).transpose(0, 1).reshape(s["case"]["hkv"], -1, D)[:, :n]
        else:
            x = _value4(s[what][p, :, :n], s[what + "s"][p, :, :n])
        out.append(x)
    return out


def _attn4(s):
    case = s["case"]
    hq, hkv, b = case["hq"], case["hkv"], case["mask"]
    for p, m in enumerate(s["new"]):
        n, a = s["lens"][p], s["starts"][p]
        k, v = _rows(s, p)
        step = max(1, (1 << 28) // (hq * n))                                 # query rows whose scores are held at once
        for i in range(0, m, step):
            r = min(step, m - i)
            q = s["qkv"][a + i:a + i + r, :hq].float().reshape(r, hkv, -1, D).permute(1, 2, 0, 3).reshape(hkv, -1, D)
            x = (q @ k.transpose(1, 2)) * (D ** -0.5)                        # [hkv][G * r][n]
            if b:
                t = n - m + i + torch.arange(r, device="cuda")
                hidden = torch.arange(n, device="cuda") >= ((t // b + 1) * b)[:, None]
                x.view(hkv, -1, r, n).masked_fill_(hidden, float("-inf"))
            top = x.amax(-1, keepdim=True)
            e = (x - top).exp_()
            total = e.sum(-1, keepdim=True)
            o = (e @ v) / total
            s["out"][a + i:a + i + r] = o.view(hkv, -1, r, D).permute(2, 0, 1, 3).reshape(r, hq, D).to(torch.bfloat16)
            s["lse"][a + i:a + i + r] = (top + total.log()).view(hkv, -1, r).permute(2, 0, 1).reshape(r, hq)
    return {"out": s["out"], "lse": s["lse"]}


# -------------------------------------------------------------------------------------------------- the library's calls
def _own(s):
    from paper_2602_14209_b200 import binding as mb
    case = s["case"]
    hq, hkv = case["hq"], case["hkv"]
    if case["op"] == "write":
        q, k, v, out = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:], {}
        if case["rope"]:
            call = {16: mb.mage_rope_append_chunk, 8: mb.mage_rope_append_chunk_kv8, 4: mb.mage_rope_append_chunk_kv4}[case["bits"]]
            call(s["kv"], s["chunk"], s["rope"], s["pos"], q, k, v, s["q_out"])
            out["q"] = s["q_out"]
        else:
            mb.mage_append_chunk_kv4(s["kv"], s["chunk"], k, v)
        if case["bits"] == 16:
            return {**out, "k": s["k"], "v": s["v"]}
        read = mb.mage_kv4_read if case["bits"] == 4 else mb.mage_kv8_read
        read(s["kv"], s["k_out"], s["v_out"], indices=s["pick"], k_eff=s["k_eff"])
        return {**out, "k": s["k_out"], "v": s["v_out"]}
    if case["op"] == "read4":
        mb.mage_kv4_read(s["kv"], s["k_out"], s["v_out"], indices=s.get("pick"), k_eff=s.get("k_eff"))
        return {"k": s["k_out"], "v": s["v_out"]}
    mb.mage_chunk_attn_kv4(s["kv"], s["chunk"], s["qkv"][:, :hq], D ** -0.5, s["out"], s["workspace"], mask_block=case["mask"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"write": _write, "read4": _read4, "attn4": _attn4}[state["case"]["op"]](state)


# -------------------------------------------------------------------------------------------- the definitions in 64 bits
def _nearest(y, grid):
    """Indexes of the points of an ascending grid nearest to y >= 0; a half goes to the even index."""
    above = torch.searchsorted(grid, y).clamp(1, grid.numel() - 1)
    below = above - 1
    up, down = grid[above] - y, y - grid[below]
    return torch.where((up < down) | ((up == down) & (above % 2 == 0)), above, below)


def _exact_value8(x):
    """The nearest e4m3 number to x * 448 / amax, times amax / 448; in 64 bits."""
    grid = torch.tensor([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:119], dtype=torch.float64, device="cuda")
    amax = x.abs().amax(-1, keepdim=True)
    scale = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
    return grid[_nearest((x / scale).abs(), grid)] * torch.sign(x) * scale


def _exact_value4(x):
    """The values that 4-bit rows of x stand for, in 64 bits: by the list of all scales and by distances."""
    scales = torch.tensor([2.0 ** (e - 17) * (1 + m / 8) for e in range(31) for m in range(8)], dtype=torch.float64, device="cuda")
    between = (scales[1:] + scales[:-1]) / 2                                 # from a half on the larger scale is taken
    g = x.reshape(-1, 16)
    s = scales[torch.searchsorted(between, g.abs().amax(-1) / 7, right=True)][:, None]
    steps = torch.arange(6, -1, -1, dtype=torch.float64, device="cuda") + 0.5
    c = (g.abs()[..., None] > steps * s[..., None]).sum(-1)                  # magnitudes beyond a half step count up, halves do not
    return (torch.sign(g) * c * s).view(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    hq, hkv, op = case["hq"], case["hkv"], case["op"]

    def place(n_rows, p):                    # of the rows n_rows of sequence p: indexes into a pool
        return (s["table"][p].long()[n_rows // case["page"]], slice(None), n_rows % case["page"]) if case["page"] else None

    def rows_of(p, what):
        n = s["lens"][p]
        j = torch.arange(n, device="cuda")
        at = place(j, p)
        code, u = (s[what][at].transpose(0, 1), s[what + "s"][at].transpose(0, 1)) if at else (s[what][p, :, :n], s[what + "s"][p, :, :n])
        w = code.reshape(code.shape[:-1] + (16, 4)).long()
        w = w[..., 0] | w[..., 1] << 8 | w[..., 2] << 16 | w[..., 3] << 24
        shift = torch.tensor([4 * (e // 2) + 16 * (e % 2) for e in range(8)], device="cuda")
        c = ((w[..., None] >> shift) & 15).reshape(code.shape[:-1] + (D,)).double() - 8
        scales = torch.tensor([2.0 ** (i // 8 - 17) * (1 + i % 8 / 8) for i in range(248)] + [math.nan] * 8, dtype=torch.float64, device="cuda")
        return c * scales[u.long()].repeat_interleave(16, -1)

    if op == "write":
        out, x = {}, s["qkv"].double()
        q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        if case["rope"]:
            turn = torch.zeros(x.shape[0], case["rot"] // 2, dtype=torch.float64, device="cuda")
            for i, a in enumerate(_axis_of_pair(case)):
                turn[:, i] = s["pos"][a].double() * s["inv_freq"][i].double()
            body = x[:, :hq + hkv, :case["rot"]]
            z = torch.complex(*(body.chunk(2, -1) if case["halves"] else (body[..., ::2].contiguous(), body[..., 1::2].contiguous())))
            z = z * torch.polar(torch.ones_like(turn), turn)[:, None]
            turned = torch.cat([z.real, z.imag], -1) if case["halves"] else torch.stack([z.real, z.imag], -1).flatten(-2)
            qk = torch.cat([turned, x[:, :hq + hkv, case["rot"]:]], -1)
            q, k = qk[:, :hq], qk[:, hq:]
            out["q"] = q
        for what, new in (("k", k), ("v", v)):
            if case["bits"] < 16:            # (what is coded is the row in 16 bits)
                val = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
                val[s["seq_of"], :, s["row_of"]] = (_exact_value8 if case["bits"] == 8 else _exact_value4)(new.bfloat16().double())
                out[what] = val
                continue
            val = torch.zeros(s[what].shape, dtype=torch.float64, device="cuda")
            for p, m in enumerate(s["new"]):
                t, rows = s["ctx"][p] + torch.arange(m, device="cuda"), slice(s["starts"][p], s["starts"][p] + m)
                at = place(t, p)
                if at:
                    val[at] = new[rows]
                else:
                    val[p].index_copy_(1, t, new[rows].transpose(0, 1))
            out[what] = val
        return out
    if op == "read4":
        out = {}
        for what in ("k", "v"):
            y = torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda")
            for p, n in enumerate(s["lens"]):
                x = rows_of(p, what)
                if case["k"]:
                    m = min(n, case["k"])
                    y[p, :, :m] = x.gather(1, s["pick"][p, :, :m, None].long().expand(-1, -1, D))
                else:
                    y[p, :, :n] = x
            out[what] = y
        return out
    if work(case)["flops"] > 5e12:
        return None
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    G = hq // hkv
    for p, m in enumerate(s["new"]):
        n, a = s["lens"][p], s["starts"][p]
        k, v = rows_of(p, "k"), rows_of(p, "v")
        t = n - m + torch.arange(m, device="cuda")
        last = torch.full_like(t, n) if case["mask"] == 0 else torch.clamp((torch.div(t, case["mask"], rounding_mode="floor") + 1) * case["mask"], max=n)
        step = max(1, (1 << 27) // n)
        for h in range(hq):
            for i in range(0, m, step):
                z = s["qkv"][a + i:a + min(m, i + step), h].double() @ k[h // G].T / math.sqrt(D)
                z[torch.arange(n, device="cuda")[None] >= last[i:i + step, None]] = -math.inf
                norm = torch.logsumexp(z, -1)
                lse[a + i:a + min(m, i + step), h] = norm
                out[a + i:a + min(m, i + step), h] = torch.exp(z - norm[:, None]) @ v[h // G]
    return {"out": out, "lse": lse}
