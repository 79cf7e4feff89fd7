"""Decode steps over a 4-bit cache held to what their arithmetic allows: one
rounding of the output, and logits of queries of any size, with channels of very
different size in one block of 32 among them (the keys are zero where the
queries are large, so the logits come from the small channels alone)."""
import numpy as np
import pytest

import q4ref
from test_gpu_q4 import BF16, F32, SCORE_RTOL, Case, store, torch, vz
from vzt import from_dev, to_dev, widen

pytestmark = pytest.mark.gpu


def check_step(c, q, kn, vn, length, left):
    """A step against the oracle.  left: what the queries' parts leave of a channel, per row of Q and block of 32
    channels.

    A logit is off by that times |k| for every channel, and by float32 sums of at most six products (2^-23 of the sum
    of the terms' magnitudes each) and two more roundings of it; p = exp(s - max) / Z carries that relative to itself,
    once for its own s and once for those in Z.  An output sum over j of p_j v_j then is off by that times the sum of
    p_j |v_j|; in a bfloat16 call by 2^-16 of it more, p being two bfloat16 numbers there, and by its one rounding to
    bfloat16, 2^-8 of it, and by 2^-18 of that sum for 64 float32 roundings."""
    m, t, gamma, d, dtype = vz(), torch(), 0.9, c.d, c.dtype
    cache, s, p = c.dev()
    out = t.zeros_like(to_dev(q))
    m.voxzip_decode_attend_score_q4(*(to_dev(x) for x in (q, kn, vn)), *cache, s, p, out, length, length, gamma,
                                    workspace=m.workspace(m.VZ_OP_DECODE_Q4, c.L, c.Hq, c.Hkv, d, c.slots))
    ref_o, ref_s, _, _ = c.expect(q, kn, vn, 0, length, length, gamma)
    K, V = (np.repeat(np.concatenate([q4ref.values(x, y)[:, :, :length],
                                      q4ref.values(*q4ref.quantise(widen(new, dtype)))[:, :, None]], 2),
                      c.Hq // c.Hkv, axis=1)
            for x, y, new in ((c.kc, c.ks, kn), (c.vc, c.vs, vn)))
    Q = widen(q, dtype)[:, :, None]
    blocks = lambda x: np.abs(x).reshape(*x.shape[:-1], -1, 32)
    cut = (left(blocks(Q).max(-1)) * blocks(K).sum(-1)).sum(-1).max()
    sums = 14 * 2.0 ** -24 * np.abs(Q * K).sum(-1).max()
    extra = 2 * d ** -0.5 * (cut + sums)
    z = (Q * K).sum(-1) * d ** -0.5
    w = np.exp(z - z.max(-1, keepdims=True))
    mean = (w[..., None] * np.abs(V)).sum(2) / w.sum(-1)[..., None]
    got_o, got_s = widen(from_dev(out), dtype), from_dev(s)
    once, parts = (2.0 ** -8, 2.0 ** -16) if dtype == BF16 else (2.0 ** -24, 0)
    assert (np.abs(got_o - ref_o) <= once * np.abs(ref_o) + (extra + parts + 2.0 ** -18) * mean).all()
    assert (np.abs(got_s - ref_s) <= (SCORE_RTOL + extra) * np.abs(ref_s)).all()


SHAPES = [(F32, 128, 8, 2), (F32, 64, 8, 1), (F32, 128, 18, 2), (F32, 64, 32, 2),
          (BF16, 128, 8, 2), (BF16, 64, 14, 2), (BF16, 128, 16, 1), (BF16, 64, 9, 1)]


# exact: small channels as multiples of 2^-13, which six parts below 2^13 hold exactly
@pytest.mark.parametrize("large,exact", [(8, False), (12, False), (12, True), (16, False)])
@pytest.mark.parametrize("length", [5, 333])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
def test_small_channels_beside_large_ones(dtype, d, Hq, Hkv, length, large, exact):
    c = Case(length + large, 2, Hq, Hkv, d, length + 1, dtype)
    K = q4ref.values(c.kc, c.ks)
    K[..., 7::32] = 0
    c.kc, c.ks = q4ref.quantise(K)
    q, kn, vn = (widen(x, dtype) for x in c.rows())
    if exact:
        q = np.round(q * 2.0 ** 13) / 2.0 ** 13
    q[..., 7::32] = (1 + c.rng.random(q[..., 7::32].shape)) * 2.0 ** large
    kn[..., 7::32] = 0
    q, kn, vn = (store(x, dtype) for x in (q, kn, vn))
    check_step(c, q, kn, vn, length, (lambda top: 0 * top) if exact else lambda top: 2.0 ** -28 * top)


@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
@pytest.mark.parametrize("power", [-112, -60, 60, 112])
def test_queries_of_any_size(dtype, d, Hq, Hkv, power):
    """Small queries on large keys and the reverse; what the parts leave is not below 2^-129."""
    c, length = Case(power + 200, 2, Hq, Hkv, d, 201, dtype), 200
    c.kc, c.ks = q4ref.quantise(q4ref.values(c.kc, c.ks) * 2.0 ** -power)
    q, kn, vn = (widen(x, dtype) for x in c.rows())
    q, kn, vn = store(q * 2.0 ** power, dtype), store(kn * 2.0 ** -power, dtype), store(vn, dtype)
    check_step(c, q, kn, vn, length, lambda top: np.maximum(2.0 ** -28 * top, 2.0 ** -129))


@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES + [(BF16, 128, 32, 4)])
@pytest.mark.parametrize("length", [0, 1, 5, 40, 700])
def test_outputs_are_rounded_once(dtype, d, Hq, Hkv, length):
    c = Case(length + 3, 2, Hq, Hkv, d, length + 1, dtype)
    check_step(c, *c.rows(), length, lambda top: 2.0 ** -28 * top)
