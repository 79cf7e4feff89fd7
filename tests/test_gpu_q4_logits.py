"""Decode steps over a 4-bit cache whose logits lie far below zero: softmax takes
the same weights from logits shifted by any amount, so heads whose every logit
is far below -128 (where 2^-logit overflows float32), or whose first keys' are,
have finite outputs and scores like any other."""
import numpy as np
import pytest

import q4ref
from test_gpu_q4 import BF16, F32, SCORE_RTOL, Case, i32, i64, store, torch, vz
from vzt import RTOL, check_close, check_rel, from_dev, to_dev, widen

pytestmark = pytest.mark.gpu

LOW = 192.0  # magnitude of K's channel 7 in keys far below the rest: logits of -134, -576 and -1536 for the heads below
HEADS = [0.0, 0.7, 3.0, 8.0]  # channel 7 of the queries, by head
SHAPES = [(BF16, 128, 8, 2), (F32, 128, 8, 2), (BF16, 64, 14, 2), (F32, 64, 8, 1),  # up to 8 heads on a KV head
          (BF16, 128, 16, 1), (F32, 128, 18, 2), (BF16, 64, 9, 1), (F32, 64, 32, 2)]  # and more
WHERE = {"all": lambda j, n: j >= 0, "first_unit": lambda j, n: j < 32, "first_half": lambda j, n: j < n // 2,
         "but_the_last": lambda j, n: j < n - 1, "in_turn": lambda j, n: j % 100 < 64}


def far_below(seed, L, Hq, Hkv, d, slots, dtype, low):
    """A cache whose keys at the slots `low` have logits far below the others', and a step's rows."""
    c = Case(seed, L, Hq, Hkv, d, slots, dtype)
    K = q4ref.values(c.kc, c.ks)
    K[..., :32] = 0
    K[:, :, low, 7] = -LOW
    c.kc, c.ks = q4ref.quantise(K)
    return c


def rows(c, n, new_low):
    """Queries, new K and V rows of n sequences [n][L][..][d]; new_low: per sequence, whether its new key is far below."""
    q, kn, vn = (widen(x, c.dtype) for x in c.rows(n))
    q[..., 7] = np.resize(HEADS, c.Hq)
    kn[..., :32] = 0
    kn[..., 7] = np.where(np.asarray(new_low), -LOW, 0)[:, None, None]
    return store(q, c.dtype), store(kn, c.dtype), store(vn, c.dtype)


def more(c, q):
    """What large logits add to the tolerance: a logit is a float32 sum of at most six products of 128 channels, each
    off by at most 2^-23 of the sum of its terms' magnitudes, then scaled and taken from the maximum, two roundings
    more; p = exp(s - max) / Z carries that relative to itself, once for its own s and once for those in Z."""
    size = (np.abs(widen(q, c.dtype)).max((0, 1, 2)) * np.abs(q4ref.values(c.kc, c.ks)).max((0, 1, 2))).sum()
    return 2 * (6 * 2 + 2) * 2.0 ** -24 * size


def check(c, got_o, got_s, ref_o, ref_s, extra, what):
    assert np.isfinite(ref_o).all() and np.isfinite(ref_s).all()
    got_o = widen(got_o, c.dtype)
    assert np.isfinite(got_o).all(), f"{what}: output"
    assert np.isfinite(got_s).all(), f"{what}: score"
    check_close(got_o, ref_o, RTOL[c.dtype] + extra, f"{what}: output")
    check_rel(got_s, ref_s, SCORE_RTOL + extra, f"{what}: score")


@pytest.mark.parametrize("where", list(WHERE))
@pytest.mark.parametrize("length", [3, 40, 390])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
def test_single(dtype, d, Hq, Hkv, length, where):
    m, t, L = vz(), torch(), 2
    low = WHERE[where](np.arange(length + 1), length + 1)
    c = far_below(length, L, Hq, Hkv, d, length + 1, dtype, low)
    q, kn, vn = (x[0] for x in rows(c, 1, low[length:]))
    extra = more(c, q[None])
    cache, s, p = c.dev()
    out = t.zeros_like(to_dev(q))
    m.voxzip_decode_attend_score_q4(*(to_dev(x) for x in (q, kn, vn)), *cache, s, p, out, length, length, 0.9,
                                    sm_scale=1.0, workspace=m.workspace(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, c.slots))
    ref_o, ref_s, _, _ = c.expect(q, kn, vn, 0, length, length, 0.9, 1.0)
    check(c, from_dev(out), from_dev(s), ref_o, ref_s, extra, where)


@pytest.mark.parametrize("dtype,d,Hq,Hkv,L,length", [(BF16, 128, 8, 2, 1, 9000), (F32, 128, 16, 1, 1, 5000),
                                                     (BF16, 64, 18, 2, 40, 700)])
@pytest.mark.parametrize("where", ["all", "first_half", "in_turn"])
def test_many_chunks(dtype, d, Hq, Hkv, L, length, where):
    m, t = vz(), torch()
    low = WHERE[where](np.arange(length + 1), length + 1)
    c = far_below(length, L, Hq, Hkv, d, length + 1, dtype, low)
    q, kn, vn = (x[0] for x in rows(c, 1, low[length:]))
    extra = more(c, q[None])
    cache, s, p = c.dev()
    out = t.zeros_like(to_dev(q))
    m.voxzip_decode_attend_score_q4(*(to_dev(x) for x in (q, kn, vn)), *cache, s, p, out, length, length, 0.9,
                                    sm_scale=1.0, workspace=m.workspace(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, c.slots))
    ref_o, ref_s, _, _ = c.expect(q, kn, vn, 0, length, length, 0.9, 1.0)
    check(c, from_dev(out), from_dev(s), ref_o, ref_s, extra, where)


@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
def test_ragged(dtype, d, Hq, Hkv):
    """A batch with a sequence of each kind."""
    m, t, L = vz(), torch(), 2
    lens = [0, 5, 700, 33, 120, 260]
    kinds = ["all"] + list(WHERE)
    base = (np.cumsum([0] + [n + 2 for n in lens])).tolist()
    total, n = base.pop(), len(lens)
    low, new_low = np.zeros(total, dtype=bool), []
    for b, ln, kind in zip(base, lens, kinds):
        low[b: b + ln + 1] = WHERE[kind](np.arange(ln + 1), ln + 1)
        new_low.append(low[b + ln])
    c = far_below(d + Hq, L, Hq, Hkv, d, total, dtype, low)
    q, kn, vn = rows(c, n, new_low)
    extra = more(c, q)
    cache, s, p = c.dev()
    out = t.zeros_like(to_dev(q))
    m.voxzip_decode_attend_score_q4_ragged(
        *(to_dev(x) for x in (q, kn, vn)), *cache, s, p, out, i64(base), i32([x + 2 for x in lens]), i32(lens), i32(lens),
        0.9, sm_scale=1.0, workspace=m.workspace_ragged(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, total, n))
    for i in range(n):
        ref_o, ref_s, _, _ = c.expect(q[i], kn[i], vn[i], base[i], lens[i], lens[i], 0.9, 1.0)
        check(c, from_dev(out)[i], from_dev(s)[:, base[i]: base[i] + lens[i] + 1], ref_o, ref_s, extra, f"{i} {kinds[i]}")


@pytest.mark.parametrize("where", ["all", "first_half"])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
def test_generation_step(dtype, d, Hq, Hkv, where):
    """The decayed scores stay finite, so the eviction in the step takes the slot of the smallest one."""
    m, t, L, length = vz(), torch(), 2, 200
    low = WHERE[where](np.arange(length + 1), length + 1)
    c = far_below(length, L, Hq, Hkv, d, length + 1, dtype, low)
    q, kn, vn = (x[0] for x in rows(c, 1, low[length:]))
    extra = more(c, q[None])
    cache, s, p = c.dev()
    out = t.zeros_like(to_dev(q))
    n = m.voxzip_decode_evict_q4(*(to_dev(x) for x in (q, kn, vn)), *cache, s, p, out, length, length + 5, 0.9, length,
                                 n_sink=2, n_recent=3, sm_scale=1.0,
                                 workspace=m.workspace(m.VZ_OP_DECODE_EVICT_Q4, L, Hq, Hkv, d, c.slots))
    assert n == length
    ref_o, ref_s, ref_p, _ = c.expect(q, kn, vn, 0, length, length + 5, 0.9, 1.0)
    pos = from_dev(p)
    of = [dict(zip(ref_p[l].tolist(), ref_s[l].tolist())) for l in range(L)]
    kept = np.array([[of[l][x] for x in pos[l, :length].tolist()] for l in range(L)])
    check(c, from_dev(out), from_dev(s)[:, :length], ref_o, kept, extra, where)
    for l in range(L):
        (gone,) = set(ref_p[l].tolist()) - set(pos[l, :length].tolist())
        compete = [v for x, v in of[l].items() if 2 <= x < length + 6 - 3]
        assert of[l][gone] <= min(compete) * (1 + 2 * (SCORE_RTOL + extra))
