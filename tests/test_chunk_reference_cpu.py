"""The rule by which a row of the prompt kernel moves the reference of its exponentials, in exact single precision on the CPU: for
logits of any size a quarter of a key tile is redone at most once, and its exponents then fit the type that P is kept in."""
import ctypes
import os
import re

import numpy as np
import pytest

F = np.float32
SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_14209_b200", "csrc", "chunk_prefill.cuh")
C = F(128 ** -0.5 * 1.4426950408889634)


def _constants(bits):
    """(kUp, kMostLog) of a cache type, as the kernel has them."""
    line = next(x for x in open(SRC) if "static constexpr float kUp" in x)
    pick = lambda name: float(re.search(name + r" = KV8 \? ([0-9.e]+)f? : ([0-9.e]+)f?", line.replace("f", "")).group(1 if bits == 8 else 2))
    return F(pick("kUp")), F(pick("kMostLog"))


def _redone(s, m, unset, up, most):
    """Times that the quarter with products s is redone under reference m, its last exponents, the last reference."""
    t = s * C                                                # rounded to single precision, like the kernel's
    for n in range(9):
        x = t - m
        if not (t.max() - m > most or unset):
            break
        m, unset = t.max() - up, False
    return n, x, m


def _rows(rng):
    for e in range(-20, 121):
        for _ in range(20):
            s = (rng.standard_normal(32) * 2.0 ** e).astype(F)
            kind = rng.integers(4)
            if kind == 0:
                s = -np.abs(s)
            elif kind == 1:                                  # close together, far from zero
                s = (F(2.0 ** e) * (1 + rng.standard_normal(32) * 2.0 ** -20)).astype(F)
            yield s, F(rng.standard_normal() * 2.0 ** rng.integers(-10, 121)), bool(rng.integers(2))


@pytest.mark.parametrize("bits", [16, 8])
def test_a_quarter_is_redone_at_most_once(bits):
    up, most = _constants(bits)
    for s, m, unset in _rows(np.random.default_rng(bits)):
        n, x, m_new = _redone(s, F(0) if unset else m, unset, up, most)
        assert n <= 1
        if n:
            assert 0 <= x.max() <= 8 and m_new <= (s * C).max()


@pytest.mark.parametrize("bits", [16, 8])
def test_the_exponent_of_the_unrounded_product_would_not_do(bits):
    """What the rounding of the logit is for: with s c - m in one fma the remainder alone, half a step of m, passes the limit, and moving
    the reference by it changes nothing."""
    up, most = _constants(bits)
    rng, stuck = np.random.default_rng(bits), 0
    for _ in range(200):
        s = (rng.standard_normal(32) * 2.0 ** 38).astype(F)
        m = F(0)
        for n in range(9):
            x = (s.astype(np.longdouble) * np.longdouble(C) - np.longdouble(m)).astype(F)
            if n and not x.max() > most:
                break
            m = F(F(m + x.max()) - up)
        stuck += n == 8
    assert stuck > 0


@pytest.mark.parametrize("scale", [float("inf"), 3e38])
def test_a_scale_that_is_not_finite_is_refused(scale):
    """Also one that is not once it is turned to powers of two.  (Nothing here reaches a GPU.)"""
    from paper_2602_14209_b200 import binding, build
    build.build()
    lib = binding.load()
    kv, chunk, kv8 = binding.mage_kv_t(), binding.mage_chunk_t(4096, 10, 5), binding.mage_kv8_t(4096, 8192, 4096, 4096)
    kv.P, kv.H_q, kv.H_kv, kv.d, kv.B, kv.N_max, kv.k_cache, kv.v_cache = 2, 8, 2, 128, 1, 2048, 4096, 4096
    kv.stride_n, kv.stride_h, kv.stride_p = 128, 2048 * 128, 2 * 2048 * 128
    p, at = ctypes.c_void_p(4096), ctypes.addressof
    assert lib.mage_chunk_attn(at(kv), at(chunk), p, 1024, 128, 1, scale, p, None, p, 1 << 40, None, None) == -1
    assert lib.mage_chunk_attn_kv8(at(kv), at(kv8), at(chunk), p, 1024, 128, 1, scale, p, None, p, 1 << 40, None, None) == -1
