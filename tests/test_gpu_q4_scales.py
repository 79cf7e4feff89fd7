"""Scale bytes at the ends of their range, those that no call writes among them:
zero-filled rows, rows of another quantiser."""
import numpy as np
import pytest

import q4ref
from test_gpu_q4 import BF16, F32, SCORE_RTOL, Case, store, torch, vz
from vzt import RTOL, check_close, check_rel, from_dev, to_dev, widen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_unpack_of_every_scale_byte_and_code(dtype, d):
    """Values past the largest float read as infinities."""
    codes = np.tile(np.r_[np.arange(16) * 17, np.arange(16) * 17], (256, d // 64)).astype(np.uint8)
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], d // 32, 1)
    out = torch().full((256, d), 3.0, dtype=torch().bfloat16 if dtype == BF16 else torch().float32, device="cuda")
    vz().voxzip_unpack_q4(to_dev(codes), to_dev(scales), out)
    want = q4ref.values(codes, scales)
    with np.errstate(over="ignore"):
        want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    assert np.array_equal(widen(from_dev(out), dtype), want, equal_nan=True)
    out.fill_(3)
    vz().voxzip_unpack_q4(to_dev(codes * 0), to_dev(scales * 0), out)
    assert not from_dev(out).any()


@pytest.mark.parametrize("byte", [0, 1, 2, 60, 200])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", [(BF16, 128, 8, 2), (F32, 128, 18, 2), (BF16, 64, 9, 1), (F32, 64, 8, 1)])
def test_decode_of_keys_of_one_scale_byte(dtype, d, Hq, Hkv, byte):
    """K's blocks at 2^(byte - 127), queries of the inverse size; the new key is zero."""
    m, t, n = vz(), torch(), 77
    c = Case(byte + d, 2, Hq, Hkv, d, n + 1, dtype)
    c.kc = c.rng.integers(0, 256, c.kc.shape).astype(np.uint8)
    c.ks[:] = byte
    q, kn, vn = (widen(x, dtype) for x in c.rows())
    q, kn, vn = store(q * 2.0 ** min(126 - byte, 125), dtype), store(kn * 0, dtype), store(vn, dtype)
    cache, s, p = c.dev()
    out = t.zeros_like(to_dev(q))
    m.voxzip_decode_attend_score_q4(*(to_dev(x) for x in (q, kn, vn)), *cache, s, p, out, n, n, 0.9,
                                    workspace=m.workspace(m.VZ_OP_DECODE_Q4, 2, Hq, Hkv, d, n + 1))
    ref_o, ref_s, _, _ = c.expect(q, kn, vn, 0, n, n, 0.9)
    # logits as in the far-below tests: at most six float32 products and two more roundings, twice
    size = np.abs(widen(q, dtype)).max() * 6 * 2.0 ** (byte - 127) * d ** 0.5
    more = 2 * 14 * 2.0 ** -24 * size
    check_close(widen(from_dev(out), dtype), ref_o, RTOL[dtype] + more, "output")
    check_rel(from_dev(s)[:, : n + 1], ref_s, SCORE_RTOL + more, "score")
