"""Host-side refusals of the calls on packed chunks: nothing here reaches a GPU."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2602_14209_b200 import build, binding
    build.build()
    return binding.load()


P = ctypes.c_void_p(4096)


def _kv(**over):
    from paper_2602_14209_b200.binding import mage_kv_t
    c = mage_kv_t()
    c.P, c.H_q, c.H_kv, c.d, c.B, c.page_size = 2, 8, 2, 128, 1, 0
    c.k_cache = c.v_cache = 4096
    c.stride_n, c.stride_h, c.stride_p, c.N_max = 128, 2048 * 128, 2 * 2048 * 128, 2048
    for k, v in over.items():
        setattr(c, k, v)
    return c


def _chunk(q_start=4096, n_tokens=10, max_len=5):
    from paper_2602_14209_b200.binding import mage_chunk_t
    return mage_chunk_t(q_start, n_tokens, max_len)


def _kv8(**over):
    from paper_2602_14209_b200.binding import mage_kv8_t
    d = dict(k8=4096, v8=8192, k_scale=4096, v_scale=4096)
    d.update(over)
    return mage_kv8_t(**d)


def _at(x):
    return None if x is None else ctypes.addressof(x)


def _attn(lib, kv, chunk, q=P, st=1024, sh=128, mask=1, scale=0.088, out=P, ws=P, ws_bytes=1 << 40):
    return lib.mage_chunk_attn(_at(kv), _at(chunk), q, st, sh, mask, scale, out, None, ws, ws_bytes, None, None)


def _attn8(lib, kv, kv8, chunk, ws_bytes=1 << 40):
    return lib.mage_chunk_attn_kv8(_at(kv), _at(kv8), _at(chunk), P, 1024, 128, 1, 0.088, P, None, P, ws_bytes, None, None)


@pytest.mark.parametrize("over,code", [(dict(d=64), -2), (dict(P=0), -1), (dict(H_q=9), -1), (dict(stride_n=100), -1), (dict(k_cache=0), -1), (dict(v_cache=4100), -2),
                                       (dict(page_size=48), -2), (dict(page_size=8), -2), (dict(page_size=64), -1), (dict(flags=1), -2), (dict(N_max=(1 << 30) + 1), -2),
                                       (dict(P=40000), -2)])
def test_cache_descriptions(lib, over, code):
    kv, ch = _kv(**over), _chunk()
    assert _attn(lib, kv, ch) == code
    assert lib.mage_append_chunk(_at(kv), _at(ch), P, P, 256, 128, None, None) == code
    if "k_cache" not in over:
        kv8 = _kv8(v8=8196) if "v_cache" in over else _kv8()
        assert _attn8(lib, kv, kv8, ch) == code
        assert lib.mage_append_chunk_kv8(_at(kv), _at(kv8), _at(ch), P, P, 256, 128, None, None) == code
        assert lib.mage_kv8_read(_at(kv), _at(kv8), None, None, 0, 8, P, P, None, None) == code


@pytest.mark.parametrize("chunk", [dict(q_start=None), dict(n_tokens=-1), dict(max_len=11), dict(max_len=-1)])
def test_chunk_descriptions(lib, chunk):
    kv, ch = _kv(), _chunk(**chunk)
    assert _attn(lib, kv, ch) == -1 and _attn(lib, kv, None) == -1
    assert lib.mage_append_chunk(_at(kv), _at(ch), P, P, 256, 128, None, None) == -1
    if "q_start" not in chunk:
        assert lib.mage_chunk_workspace_bytes(_at(kv), _at(ch)) == 0


def test_arguments_of_the_attention(lib):
    kv, ch = _kv(), _chunk()
    need = lib.mage_chunk_workspace_bytes(_at(kv), _at(ch))
    assert need > 0 and need % 256 == 0 and lib.mage_chunk_workspace_bytes(_at(None), _at(ch)) == 0 and lib.mage_chunk_workspace_bytes(_at(kv), _at(None)) == 0
    assert _attn(lib, kv, ch, ws_bytes=need - 1) == -3
    assert _attn(lib, kv, ch, q=None) == -1 and _attn(lib, kv, ch, out=None) == -1 and _attn(lib, kv, ch, ws=None) == -1
    assert _attn(lib, kv, ch, ws=ctypes.c_void_p(4097 + 15)) == -1
    assert _attn(lib, kv, ch, mask=-1) == -1 and _attn(lib, kv, ch, scale=0.0) == -1 and _attn(lib, kv, ch, scale=float("nan")) == -1
    assert _attn(lib, kv, ch, st=1020) == -1 and _attn(lib, kv, ch, sh=-128) == -1
    assert _attn(lib, kv, ch, q=ctypes.c_void_p(4098)) == -2 and _attn(lib, kv, ch, out=ctypes.c_void_p(4104)) == -2
    assert _attn(lib, None, ch) == -1
    assert _attn(lib, kv, _chunk(n_tokens=0, max_len=0)) == 0            # nothing to do: no launch
    assert _attn8(lib, kv, None, ch) == -1
    assert _attn8(lib, kv, _kv8(k8=None), ch) == -1 and _attn8(lib, kv, _kv8(v_scale=None), ch) == -1 and _attn8(lib, kv, _kv8(k8=4104), ch) == -2
    assert _attn8(lib, _kv(stride_n=136, stride_h=2048 * 136, stride_p=4096 * 136), _kv8(), ch) == -2
    assert _attn8(lib, kv, _kv8(), ch, ws_bytes=16) == -3


def test_workspace_covers_both_cache_types_and_stays_small(lib):
    for n, m in ((1, 1), (64, 1), (5000, 4096)):
        for N in (0, 100, 131072, 1 << 20):
            kv = _kv(P=64, H_q=32, H_kv=8, N_max=N, stride_h=max(N, 1) * 128, stride_p=8 * max(N, 1) * 128)
            assert 0 < lib.mage_chunk_workspace_bytes(_at(kv), _at(_chunk(n_tokens=n, max_len=m))) < 1 << 30


def test_arguments_of_the_cache_calls(lib):
    kv, ch = _kv(), _chunk()
    assert lib.mage_append_chunk(_at(kv), _at(ch), None, P, 256, 128, None, None) == -1 and lib.mage_append_chunk(_at(kv), _at(ch), P, None, 256, 128, None, None) == -1
    assert lib.mage_append_chunk(_at(kv), _at(ch), P, P, 255, 128, None, None) == -1 and lib.mage_append_chunk(_at(kv), _at(ch), ctypes.c_void_p(4104), P, 256, 128, None, None) == -2
    assert lib.mage_append_chunk_kv8(_at(kv), _at(None), _at(ch), P, P, 256, 128, None, None) == -1
    for over in (dict(stride_h=0), dict(stride_p=0)):                       # heads or problems that share memory
        assert lib.mage_append_chunk(_at(_kv(**over)), _at(ch), P, P, 256, 128, None, None) == -1
        assert lib.mage_append_chunk_kv8(_at(_kv(**over)), _at(_kv8()), _at(ch), P, P, 256, 128, None, None) == -1
    k8 = _kv8()
    assert lib.mage_kv8_read(_at(kv), _at(k8), None, None, -1, 8, P, P, None, None) == -1 and lib.mage_kv8_read(_at(kv), _at(k8), None, None, 0, -1, P, P, None, None) == -1
    assert lib.mage_kv8_read(_at(kv), _at(k8), P, None, 0, 8, P, P, None, None) == -1 and lib.mage_kv8_read(_at(kv), _at(k8), P, P, 3, 8, P, P, None, None) == -1
    assert lib.mage_kv8_read(_at(kv), _at(k8), None, None, 0, 8, None, P, None, None) == -1 and lib.mage_kv8_read(_at(kv), _at(k8), None, None, 0, 8, P, ctypes.c_void_p(4104), None, None) == -2
    assert lib.mage_kv8_read(_at(kv), _at(None), None, None, 0, 8, P, P, None, None) == -1
    assert lib.mage_kv8_read(_at(kv), _at(k8), None, None, 0, 0, P, P, None, None) == 0


def test_arguments_of_the_rotation(lib):
    from paper_2602_14209_b200.binding import mage_rope_t

    def call(q=P, qs=(1024, 128), k=P, ks=(256, 128), qo=ctypes.c_void_p(8192), qos=(1024, 128), ko=ctypes.c_void_p(16384), kos=(256, 128), axis=0, n_tokens=4, H_q=8,
             H_kv=2, positions=P, pos_stride=4, **over):
        d = dict(d=128, rot_dim=128, halves=1, n_axes=1, mult=1.0, inv_freq=4096)
        d.update(over)
        r = mage_rope_t(**d)
        r.axis_of_pair[3] = axis
        return lib.mage_rope(ctypes.addressof(r), n_tokens, positions, pos_stride, H_q, q, *qs, qo, *qos, H_kv, k, *ks, ko, *kos, None)

    assert call(d=64, rot_dim=64) == -2 and call(rot_dim=24) == -2 and call(rot_dim=144) == -1 and call(rot_dim=0) == -1
    assert call(n_axes=0) == -1 and call(n_axes=5) == -2 and call(axis=1) == -1 and call(n_tokens=-1) == -1 and call(H_q=0) == -1
    assert call(positions=None) == -1 and call(inv_freq=None) == -1 and call(q=None) == -1 and call(k=None) == -1 and call(ko=None) == -1
    assert call(mult=float("inf")) == -1 and call(qs=(1020, 128)) == -1 and call(kos=(-8, 128)) == -1
    assert call(q=ctypes.c_void_p(4104)) == -2 and call(ko=ctypes.c_void_p(4104)) == -2
    assert call(qo=P, qos=(2048, 128)) == -1                             # in place under other strides
    for over in (dict(qos=(0, 128)), dict(qos=(1024, 64)), dict(kos=(64, 128)), dict(kos=(256, 0))):
        assert call(**over) == -1                                        # outputs that share memory
    assert call(n_tokens=0) == 0
    assert lib.mage_rope(None, 4, P, 4, 8, P, 0, 0, P, 0, 0, 2, P, 0, 0, P, 0, 0, None) == -1


def test_the_binding_checks_its_tensors(lib):
    from paper_2602_14209_b200 import binding as mb
    z8, s = torch.zeros(2, 2, 16, 128, dtype=torch.uint8), torch.zeros(2, 2, 16)
    kv8 = mb.Kv8Cache(z8, z8.clone(), s, s.clone(), 4)
    assert kv8.N_max == 16 and kv8.P == 2
    with pytest.raises(ValueError):
        mb.Kv8Cache(z8, z8, s[:, :1], s, 4)
    with pytest.raises(ValueError):
        mb.Kv8Cache(z8.bfloat16(), z8, s, s, 4)
    with pytest.raises(ValueError):
        mb.ChunkBatch(kv8, torch.zeros(2, dtype=torch.int32), 1)
    with pytest.raises(ValueError):
        mb.ChunkBatch(kv8, torch.zeros(3, dtype=torch.int32), 1, max_len=2)
    chunk = mb.ChunkBatch(kv8, torch.zeros(3, dtype=torch.int32), 3)
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mb.mage_append_chunk_kv8(kv8, chunk, x[:2], x)
    with pytest.raises(ValueError):
        mb.mage_chunk_attn_kv8(kv8, chunk, x, 1.0, x, torch.zeros(8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        mb.mage_kv8_read(kv8, x, x)
    with pytest.raises(ValueError):
        mb.Rope(torch.zeros(64), axis_of_pair=[0] * 63)
    rope = mb.Rope(torch.zeros(64), axis_of_pair=[0] * 63 + [1])
    with pytest.raises(ValueError):
        mb.mage_rope(rope, torch.zeros(1, 3, dtype=torch.int32), x)
