"""Host-side refusals of the calls over a 4-bit cache and of the writes that rotate: nothing here reaches a GPU."""
import ctypes

import pytest
import torch

from test_abi_chunk_cpu import P, _at, _chunk, _kv, _kv8, lib  # noqa: F401


def _kv4(**over):
    from paper_2602_14209_b200.binding import mage_kv4_t
    d = dict(k4=4096, v4=8192, k_scale=4096, v_scale=8192)
    d.update(over)
    return mage_kv4_t(**d)


def _rope(**over):
    from paper_2602_14209_b200.binding import mage_rope_t
    axis = over.pop("axis", 0)
    d = dict(d=128, rot_dim=128, halves=1, n_axes=1, mult=1.0, inv_freq=4096)
    d.update(over)
    r = mage_rope_t(**d)
    r.axis_of_pair[3] = axis
    return r


def _attn4(lib, kv, kv4, chunk, q=P, st=1024, sh=128, mask=1, scale=0.088, out=P, ws=P, ws_bytes=1 << 40):
    return lib.mage_chunk_attn_kv4(_at(kv), _at(kv4), _at(chunk), q, st, sh, mask, scale, out, None, ws, ws_bytes, None, None)


def _append4(lib, kv, kv4, chunk, k=P, v=P, st=256, sh=128):
    return lib.mage_append_chunk_kv4(_at(kv), _at(kv4), _at(chunk), k, v, st, sh, None, None)


def _read4(lib, kv, kv4, indices=None, k_eff=None, begin=0, n=8, k=P, v=P):
    return lib.mage_kv4_read(_at(kv), _at(kv4), indices, k_eff, begin, n, k, v, None, None)


def _rotate(lib, kv, codes, chunk, bits=4, rope=None, pos=P, pos_stride=10, q=P, qs=(1024, 128), qo=ctypes.c_void_p(1 << 20), qos=(1024, 128), k=P, v=P, ks=(256, 128)):
    rope = _rope() if rope is None else rope
    args = (_at(chunk), _at(rope), pos, pos_stride, q, *qs, qo, *qos, k, v, *ks, None, None)
    if bits == 16:
        return lib.mage_rope_append_chunk(_at(kv), *args)
    return (lib.mage_rope_append_chunk_kv8 if bits == 8 else lib.mage_rope_append_chunk_kv4)(_at(kv), _at(codes), *args)


@pytest.mark.parametrize("over,code", [(dict(d=64), -2), (dict(P=0), -1), (dict(H_q=9), -1), (dict(stride_n=100), -1), (dict(page_size=48), -2), (dict(page_size=8), -2),
                                       (dict(page_size=64), -1), (dict(flags=1), -2), (dict(N_max=(1 << 30) + 1), -2), (dict(P=40000), -2), (dict(stride_n=144), -2),
                                       (dict(stride_h=2048 * 128 + 16), -2)])
def test_cache_descriptions(lib, over, code):
    kv, ch = _kv(**over), _chunk()
    assert _attn4(lib, kv, _kv4(), ch) == code and _append4(lib, kv, _kv4(), ch) == code and _read4(lib, kv, _kv4()) == code and _rotate(lib, kv, _kv4(), ch) == code
    if "stride" not in str(over):
        assert _rotate(lib, kv, _kv8(), ch, 8) == code and _rotate(lib, kv, None, ch, 16) == code


@pytest.mark.parametrize("over,code", [(dict(k4=None), -1), (dict(v4=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1), (dict(k4=4104), -2), (dict(v4=4100), -2),
                                       (dict(k_scale=4104), -2), (dict(v_scale=4097), -2)])
def test_code_arrays(lib, over, code):
    kv, ch, kv4 = _kv(), _chunk(), _kv4(**over)
    assert _attn4(lib, kv, kv4, ch) == code and _append4(lib, kv, kv4, ch) == code and _read4(lib, kv, kv4) == code and _rotate(lib, kv, kv4, ch) == code
    assert _attn4(lib, kv, None, ch) == -1 and _append4(lib, kv, None, ch) == -1 and _read4(lib, kv, None) == -1 and _rotate(lib, kv, None, ch) == -1
    assert _rotate(lib, kv, None, ch, 8) == -1 and _attn4(lib, None, _kv4(), ch) == -1


@pytest.mark.parametrize("chunk", [dict(q_start=None), dict(n_tokens=-1), dict(max_len=11), dict(max_len=-1)])
def test_chunk_descriptions(lib, chunk):
    ch = _chunk(**chunk)
    assert _attn4(lib, _kv(), _kv4(), ch) == -1 and _append4(lib, _kv(), _kv4(), ch) == -1
    for bits, codes in ((16, None), (8, _kv8()), (4, _kv4())):
        assert _rotate(lib, _kv(), codes, ch, bits) == -1 and _rotate(lib, _kv(), codes, None, bits) == -1


def test_arguments_of_attention_write_and_read(lib):
    kv, ch, kv4 = _kv(), _chunk(), _kv4()
    need = lib.mage_chunk_workspace_bytes(_at(kv), _at(ch))
    assert _attn4(lib, kv, kv4, ch, ws_bytes=need - 1) == -3
    assert _attn4(lib, kv, kv4, ch, q=None) == -1 and _attn4(lib, kv, kv4, ch, out=None) == -1 and _attn4(lib, kv, kv4, ch, ws=None) == -1
    assert _attn4(lib, kv, kv4, ch, mask=-1) == -1 and _attn4(lib, kv, kv4, ch, scale=0.0) == -1 and _attn4(lib, kv, kv4, ch, scale=float("inf")) == -1
    assert _attn4(lib, kv, kv4, ch, st=1020) == -1 and _attn4(lib, kv, kv4, ch, q=ctypes.c_void_p(4098)) == -2
    assert _append4(lib, kv, kv4, ch, k=None) == -1 and _append4(lib, kv, kv4, ch, v=ctypes.c_void_p(4104)) == -2 and _append4(lib, kv, kv4, ch, st=255) == -1
    for over in (dict(stride_h=0), dict(stride_p=0)):
        assert _append4(lib, _kv(**over), kv4, ch) == -1 and _rotate(lib, _kv(**over), kv4, ch) == -1 and _rotate(lib, _kv(**over), None, ch, 16) == -1
    assert _read4(lib, kv, kv4, begin=-1) == -1 and _read4(lib, kv, kv4, n=-1) == -1 and _read4(lib, kv, kv4, indices=P) == -1 and _read4(lib, kv, kv4, P, P, 3) == -1
    assert _read4(lib, kv, kv4, k=None) == -1 and _read4(lib, kv, kv4, v=ctypes.c_void_p(4104)) == -2 and _read4(lib, kv, kv4, n=0) == 0
    empty = _chunk(n_tokens=0, max_len=0)                                # nothing to do: no launch
    assert _attn4(lib, kv, kv4, empty) == 0 and _append4(lib, kv, kv4, empty) == 0 and _rotate(lib, kv, kv4, empty) == 0


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_arguments_of_the_rotation(lib, bits):
    kv, ch, codes = _kv(), _chunk(), {16: None, 8: _kv8(), 4: _kv4()}[bits]

    def call(**over):
        return _rotate(lib, kv, codes, ch, bits, **over)

    assert call(rope=_rope(d=64, rot_dim=64)) == -2 and call(rope=_rope(rot_dim=24)) == -2 and call(rope=_rope(rot_dim=144)) == -1 and call(rope=_rope(rot_dim=0)) == -1
    assert call(rope=_rope(n_axes=0)) == -1 and call(rope=_rope(n_axes=5)) == -2 and call(rope=_rope(axis=1)) == -1 and call(rope=_rope(inv_freq=None)) == -1
    assert call(rope=_rope(mult=float("nan"))) == -1
    assert call(pos=None) == -1 and call(pos_stride=-1) == -1 and call(q=None) == -1 and call(qo=None) == -1 and call(k=None) == -1 and call(v=None) == -1
    assert call(qs=(1020, 128)) == -1 and call(qos=(1024, -8)) == -1 and call(ks=(256, 100)) == -1
    for name in ("q", "qo", "k", "v"):
        assert call(**{name: ctypes.c_void_p(4104)}) == -2
    assert call(qo=P, qos=(2048, 128)) == -1                             # in place under other strides
    assert call(qos=(0, 128)) == -1 and call(qos=(1024, 64)) == -1       # outputs that share memory


def test_the_binding_checks_its_tensors(lib):
    from paper_2602_14209_b200 import binding as mb
    z, s = torch.zeros(2, 2, 16, 64, dtype=torch.uint8), torch.zeros(2, 2, 16, 8, dtype=torch.uint8)
    kv4 = mb.Kv4Cache(z, z.clone(), s, s.clone(), 4)
    assert kv4.N_max == 16 and kv4.P == 2 and kv4.d == 128 and kv4.c.stride_n == 128 and kv4.c.stride_p == 2 * 16 * 128
    like = mb.Kv4Cache.like(mb.KVCache(torch.zeros(2, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 16, 128, dtype=torch.bfloat16), 4, 1))
    assert tuple(like.k4.shape) == (2, 2, 16, 64) and tuple(like.v_scale.shape) == (2, 2, 16, 8)
    for bad in ((z, z, s[:, :1], s), (z.int(), z, s, s), (z, z[:, :, :8], s, s), (z, z, s.float(), s)):
        with pytest.raises(ValueError):
            mb.Kv4Cache(*bad, 4)
    chunk = mb.ChunkBatch(kv4, torch.zeros(3, dtype=torch.int32), 3)
    x, q = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mb.mage_append_chunk_kv4(kv4, chunk, x[:2], x)
    with pytest.raises(ValueError):
        mb.mage_chunk_attn_kv4(kv4, chunk, x, 1.0, x, torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        mb.mage_kv4_read(kv4, x, x)
    rope, pos = mb.Rope(torch.zeros(64)), torch.zeros(3, dtype=torch.int32)
    for args in ((pos[:2], q, x, x), (pos, q[:2], x, x), (pos, q, x, x.float()), (pos.long(), q, x, x), (pos, q, x, x, q[:, :2])):
        with pytest.raises(ValueError):
            mb.mage_rope_append_chunk_kv4(kv4, chunk, rope, *args)


def test_workspace_for_the_copy(lib):
    """Room for a 16-bit copy of the cache with prompts, none for few tokens or for very large batches; the attention takes the smaller size, too."""
    size, more = lib.mage_chunk_workspace_bytes, lib.mage_chunk_workspace_bytes_kv4
    kv = _kv(P=1, H_q=28, H_kv=4, N_max=40000, stride_h=40000 * 128, stride_p=160000 * 128)
    for n, copies in ((1, False), (40, False), (89, False), (90, True), (4096, True)):
        ch = _chunk(n_tokens=n, max_len=n)
        assert more(_at(kv), _at(ch)) == size(_at(kv), _at(ch)) + (2 * 40000 * 4 * 256 if copies else 0)
    big = _kv(P=64, H_q=32, H_kv=8, N_max=131072, stride_h=131072 * 128, stride_p=8 * 131072 * 128)
    ch = _chunk(n_tokens=64 * 2000, max_len=2000)
    assert more(_at(big), _at(ch)) == size(_at(big), _at(ch))
    assert more(_at(_kv(d=64)), _at(ch)) == 0 and more(None, _at(ch)) == 0 and more(_at(kv), None) == 0
    assert _attn4(lib, kv, _kv4(), _chunk(n_tokens=4096, max_len=4096), ws_bytes=size(_at(kv), _at(_chunk(n_tokens=4096, max_len=4096))) - 1) == -3


@pytest.mark.parametrize("made_for", ["16", "8", "4"])
def test_the_binding_refuses_a_cache_of_another_kind(lib, made_for):
    """Calls over codes take the cache class whose codes and scales they address: anything else would be read or written behind its arrays."""
    from paper_2602_14209_b200 import binding as mb
    rows = torch.zeros(2, 2, 16, 128, dtype=torch.bfloat16)
    kv16 = mb.KVCache(rows, rows.clone(), 4, 1)
    caches = {"16": kv16, "8": mb.Kv8Cache.like(kv16), "4": mb.Kv4Cache.like(kv16)}
    kv = caches[made_for]
    chunk = mb.ChunkBatch(kv, torch.zeros(3, dtype=torch.int32), 3)
    x, q = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    out, ws, rope, pos = torch.zeros(2, 2, 8, 128, dtype=torch.bfloat16), torch.zeros(1 << 20, dtype=torch.uint8), mb.Rope(torch.zeros(64)), torch.zeros(3, dtype=torch.int32)
    for kind in ("8", "4"):
        if kind == made_for:
            continue
        calls = ((f"mage_append_chunk_kv{kind}", (chunk, x, x)), (f"mage_kv{kind}_read", (out, out.clone())), (f"mage_chunk_attn_kv{kind}", (chunk, q, 0.1, torch.zeros_like(q), ws)),
                 (f"mage_rope_append_chunk_kv{kind}", (chunk, rope, pos, q, x, x)))
        for name, args in calls:
            with pytest.raises(ValueError, match=f"Kv{kind}Cache"):
                getattr(mb, name)(kv, *args)


@pytest.mark.parametrize("kind", ["Kv8Cache", "Kv4Cache"])
def test_a_coded_cache_like_one_whose_tensors_have_spare_rows(lib, kind):
    """A 16-bit cache may use fewer rows than its tensors have: the coded one has those it uses, and so the same lengths."""
    from paper_2602_14209_b200 import binding as mb
    rows = torch.zeros(2, 3, 40, 128, dtype=torch.bfloat16)
    kv = mb.KVCache(rows, rows.clone(), 6, 4, N_max=25)
    like = getattr(mb, kind).like(kv)
    assert (like.N_max, like.P, like.H_q, like.H_kv, like.B) == (25, 2, 6, 3, 4) and like.c.N_max == 25 and tuple(like.k_scale.shape[:3]) == (2, 3, 25)
    table = torch.zeros(2, 3, dtype=torch.int32)
    paged = mb.KVCache(rows[:, :, :16].contiguous(), rows[:, :, :16].contiguous(), 6, 4, block_table=table, N_max=25)
    like = getattr(mb, kind).like(paged)
    assert like.N_max == 25 and tuple(like.k_scale.shape[:3]) == (2, 3, 16) and like.c.num_pages == 2


@pytest.mark.parametrize("G,per", [(1, 640), (4, 160), (7, 90), (16, 40), (128, 5)])
def test_from_where_on_there_is_room_for_the_copy(lib, G, per):
    """5 * (128 / G) new tokens a problem on average, however they are spread."""
    size, more = lib.mage_chunk_workspace_bytes, lib.mage_chunk_workspace_bytes_kv4
    kv = _kv(P=3, H_q=2 * G, H_kv=2)
    for n, copies in ((3 * per - 1, False), (3 * per, True)):
        for most in (-(-n // 3), n):
            ch = _chunk(n_tokens=n, max_len=most)
            assert more(_at(kv), _at(ch)) == size(_at(kv), _at(ch)) + (2 * 3 * 2 * 2048 * 256 if copies else 0)
