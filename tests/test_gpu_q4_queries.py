"""Queries with channels of very different size in one block of 32, over a 4-bit
cache whose keys are zero where the queries are large: the logits come from the
small channels alone."""
import numpy as np
import pytest

import q4ref
from test_gpu_q4 import BF16, F32, SCORE_RTOL, Case, store, torch, vz
from vzt import RTOL, from_dev, to_dev, widen

pytestmark = pytest.mark.gpu


# exact: small channels as multiples of 2^-13, which six parts below 2^13 hold exactly
@pytest.mark.parametrize("large,exact", [(8, False), (12, False), (12, True), (16, False)])
@pytest.mark.parametrize("length", [5, 333])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", [(F32, 128, 8, 2), (F32, 64, 8, 1), (F32, 128, 18, 2), (F32, 64, 32, 2),
                                            (BF16, 128, 8, 2), (BF16, 64, 14, 2), (BF16, 128, 16, 1), (BF16, 64, 9, 1)])
def test_small_channels_beside_large_ones(dtype, d, Hq, Hkv, length, large, exact):
    m, t, L, gamma = vz(), torch(), 2, 0.9
    c = Case(length + large, L, Hq, Hkv, d, length + 1, dtype)
    K = q4ref.values(c.kc, c.ks)
    K[..., 7::32] = 0
    c.kc, c.ks = q4ref.quantise(K)
    q, kn, vn = (widen(x, dtype) for x in c.rows())
    if exact:
        q = np.round(q * 2.0 ** 13) / 2.0 ** 13
    q[..., 7::32] = (1 + c.rng.random(q[..., 7::32].shape)) * 2.0 ** large
    kn[..., 7::32] = 0
    q, kn, vn = (store(x, dtype) for x in (q, kn, vn))
    cache, s, p = c.dev()
    out = t.zeros_like(to_dev(q))
    m.voxzip_decode_attend_score_q4(*(to_dev(x) for x in (q, kn, vn)), *cache, s, p, out, length, length, gamma,
                                    workspace=m.workspace(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, c.slots))
    ref_o, ref_s, _, _ = c.expect(q, kn, vn, 0, length, length, gamma)
    # A logit is off by what the queries' parts leave, 2^-28 of a block's largest channel per channel, and by float32
    # sums of at most six products (2^-23 of the sum of the terms' magnitudes each) and two more roundings of it;
    # p = exp(s - max) / Z carries that relative to itself, once for its own s and once for those in Z.  An output
    # sum over j of p_j v_j then is off by that times the sum of p_j |v_j|.
    new = [q4ref.values(*q4ref.quantise(widen(x, dtype)))[:, :, None] for x in (kn, vn)]
    K, V = (np.repeat(np.concatenate([x[:, :, :length], y], 2), Hq // Hkv, axis=1)
            for x, y in ((K, new[0]), (q4ref.values(c.vc, c.vs), new[1])))
    Q = widen(q, dtype)[:, :, None]
    blocks = lambda x: np.abs(x).reshape(*x.shape[:-1], -1, 32)
    left = 0 if exact else 2.0 ** -28 * (blocks(Q).max(-1) * blocks(K).sum(-1)).sum(-1).max()
    sums = 14 * 2.0 ** -24 * np.abs(Q * K).sum(-1).max()
    extra = 2 * d ** -0.5 * (left + sums)
    z = (Q * K).sum(-1) * d ** -0.5
    w = np.exp(z - z.max(-1, keepdims=True))
    mean = (w[..., None] * np.abs(V)).sum(2) / w.sum(-1)[..., None]
    got_o, got_s = widen(from_dev(out), dtype), from_dev(s)
    rms = np.sqrt((ref_o ** 2).mean(-1, keepdims=True))
    assert (np.abs(got_o - ref_o) <= RTOL[dtype] * (np.abs(ref_o) + rms) + extra * mean).all()
    assert (np.abs(got_s - ref_s) <= (SCORE_RTOL + extra) * np.abs(ref_s)).all()
