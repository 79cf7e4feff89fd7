"""The 4-bit cache without a GPU: the reference's own rounding against brute
force, and what the entry points refuse on the host."""
import ctypes

import numpy as np
import pytest

import paper_2608_08569_amd as vz
import q4ref

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: every case fails validation first
OFF8 = ctypes.c_void_p(0x10008)
ODD = ctypes.c_void_p(0x10001)


def test_reference_picks_the_nearest_value_and_the_smallest_scale():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 64)) * 2.0 ** rng.integers(-20, 20, (200, 1))
    x[:50] = rng.integers(-28, 29, (50, 64)) / 4  # borders and ties
    x[50] = 0
    codes, scales = q4ref.quantise(x)
    v = q4ref.values(codes, scales)
    grid = np.concatenate([q4ref.MAG, -q4ref.MAG])
    e = scales.astype(int) - 127
    unit = np.repeat(2.0 ** e, 32, axis=-1)
    best = np.abs(x[..., None] - grid * unit[..., None]).min(-1)
    assert np.array_equal(np.abs(x - v), best)  # differences of these values are exact
    top = np.abs(x).reshape(200, 2, 32).max(-1)
    assert np.all(top <= 7 * 2.0 ** e)
    assert np.all((top > 7 * 2.0 ** (e - 1)) | (e == -125))
    ties = q4ref.quantise(np.array([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5] + [0.0] * 24))[0][:4]
    assert ties.tolist() == [0x07, 0x22, 0x44, 0x66]  # to the even code
    assert q4ref.quantise(np.full(32, 7.0))[1][0] == 127 and q4ref.quantise(np.full(32, 7.5))[1][0] == 128


def _fuse(**kw):
    at = lambda x: ctypes.c_void_p(x << 20)
    a = dict(ki=at(1), vi=at(2), T=100, off=FAKE, n=30, ak=None, av=None, kc=at(3), ks=at(4), vc=at(5), vs=at(6),
             so=FAKE, po=FAKE, L=1, H=1, d=64, cap=32, dtype=vz.VZ_F32)
    a.update(kw)
    return vz.lib().voxzip_fuse_spans_q4(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(off=None), vz.VZ_ERR_INVALID), (dict(vi=None), vz.VZ_ERR_INVALID), (dict(ks=None), vz.VZ_ERR_INVALID),
    (dict(ak=FAKE), vz.VZ_ERR_INVALID), (dict(kc=ctypes.c_void_p(0x100040)), vz.VZ_ERR_INVALID),
    (dict(vs=ctypes.c_void_p(0x400004)), vz.VZ_ERR_INVALID),   # v_scales inside k_scales
    (dict(vc=OFF8), vz.VZ_ERR_INVALID), (dict(ks=ODD), vz.VZ_ERR_INVALID),
    (dict(n=33), vz.VZ_ERR_CAPACITY), (dict(n=101, cap=200), vz.VZ_ERR_SHAPE),
    (dict(d=256), vz.VZ_ERR_UNSUPPORTED),                      # wide rows stay in full precision
    (dict(d=96), vz.VZ_ERR_UNSUPPORTED), (dict(dtype=2), vz.VZ_ERR_UNSUPPORTED), (dict(H=40000), vz.VZ_ERR_UNSUPPORTED),
    (dict(L=0), vz.VZ_ERR_SHAPE),
])
def test_fuse_q4_rejects(kw, code):
    assert _fuse(**kw) == code
    assert vz.lib().voxzip_last_error().decode().startswith("voxzip_fuse_spans_q4")


def test_fuse_q4_ragged_rejects():
    at = lambda x: ctypes.c_void_p(x << 20)
    base = dict(ki=at(1), vi=at(2), ib=FAKE, T=FAKE, total_in=100, off=FAKE, ob=FAKE, n=FAKE, total_off=31, most=30,
                ak=None, av=None, kc=at(3), ks=at(4), vc=at(5), vs=at(6), so=FAKE, po=FAKE, b=FAKE, cap=FAKE,
                total=64, S=2, status=None, L=1, H=1, d=128, dtype=vz.VZ_BF16)
    for kw, code in ((dict(b=None), vz.VZ_ERR_INVALID), (dict(av=FAKE), vz.VZ_ERR_INVALID),
                     (dict(kc=OFF8), vz.VZ_ERR_INVALID), (dict(S=0), vz.VZ_ERR_SHAPE), (dict(total=0), vz.VZ_ERR_SHAPE),
                     (dict(most=65), vz.VZ_ERR_SHAPE), (dict(d=32), vz.VZ_ERR_UNSUPPORTED),
                     (dict(total=1 << 26, most=1 << 26, S=8), vz.VZ_ERR_UNSUPPORTED)):
        assert vz.lib().voxzip_fuse_spans_q4_ragged(*{**base, **kw}.values(), None) == code, kw


@pytest.mark.parametrize("kw,code", [
    (dict(codes=None), vz.VZ_ERR_INVALID), (dict(codes=ODD), vz.VZ_ERR_INVALID), (dict(out=OFF8), vz.VZ_ERR_INVALID),
    (dict(out=FAKE), vz.VZ_ERR_INVALID), (dict(n=-1), vz.VZ_ERR_SHAPE), (dict(n=(1 << 28) + 1), vz.VZ_ERR_SHAPE),
    (dict(d=32), vz.VZ_ERR_UNSUPPORTED), (dict(dtype=5), vz.VZ_ERR_UNSUPPORTED),
])
def test_unpack_q4_rejects(kw, code):
    a = dict(codes=FAKE, scales=ctypes.c_void_p(0x800000), n=4, d=128, out=ctypes.c_void_p(0x900000), dtype=vz.VZ_BF16)
    a.update(kw)
    assert vz.lib().voxzip_unpack_q4(*a.values(), None) == code


DECODE = [
    (dict(q=None), vz.VZ_ERR_INVALID), (dict(ks=None), vz.VZ_ERR_INVALID), (dict(vs=None), vz.VZ_ERR_INVALID),
    (dict(kc=OFF8), vz.VZ_ERR_INVALID), (dict(vs=ODD), vz.VZ_ERR_INVALID), (dict(gamma=1.5), vz.VZ_ERR_INVALID),
    (dict(gamma=float("nan")), vz.VZ_ERR_INVALID), (dict(scale=float("inf")), vz.VZ_ERR_INVALID),
    (dict(Hq=30), vz.VZ_ERR_SHAPE), (dict(L=0), vz.VZ_ERR_SHAPE), (dict(Hq=68), vz.VZ_ERR_UNSUPPORTED),
    (dict(Hq=320, Hkv=20), vz.VZ_ERR_UNSUPPORTED), (dict(d=96), vz.VZ_ERR_UNSUPPORTED),
    (dict(dtype=7), vz.VZ_ERR_UNSUPPORTED), (dict(ws=None), vz.VZ_ERR_WORKSPACE),
    (dict(ws_bytes=16), vz.VZ_ERR_WORKSPACE), (dict(ws=OFF8), vz.VZ_ERR_WORKSPACE),
]
COMMON = dict(q=FAKE, kn=FAKE, vn=FAKE, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, s=FAKE, p=FAKE, o=FAKE)


@pytest.mark.parametrize("kw,code", DECODE + [(dict(len=-1), vz.VZ_ERR_INVALID), (dict(len=64), vz.VZ_ERR_CAPACITY)])
def test_decode_q4_rejects(kw, code):
    a = dict(COMMON, len=10, next_pos=10, gamma=0.95, scale=0.0, L=2, Hq=32, Hkv=4, d=128, cap=64, dtype=vz.VZ_BF16,
             ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    assert vz.lib().voxzip_decode_attend_score_q4(*a.values(), None) == code
    assert vz.lib().voxzip_last_error().decode().startswith("voxzip_decode_attend_score_q4")


@pytest.mark.parametrize("kw,code", DECODE + [
    (dict(len=64), vz.VZ_ERR_CAPACITY), (dict(budget=0), vz.VZ_ERR_INVALID), (dict(sink=60), vz.VZ_ERR_INVALID),
    (dict(next_pos=(1 << 31) - 1), vz.VZ_ERR_INVALID), (dict(kept=FAKE, next_pos=1 << 18), vz.VZ_ERR_UNSUPPORTED)])
def test_decode_evict_q4_rejects(kw, code):
    n = ctypes.c_int32(-7)
    a = dict(COMMON, len=10, next_pos=10, gamma=0.95, scale=0.0, budget=10, sink=4, recent=-1, kept=None,
             new=ctypes.byref(n), L=2, Hq=32, Hkv=4, d=128, cap=64, dtype=vz.VZ_BF16, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    assert vz.lib().voxzip_decode_evict_q4(*a.values(), None) == code
    assert n.value == -7


@pytest.mark.parametrize("kw,code", DECODE + [(dict(b=None), vz.VZ_ERR_INVALID), (dict(S=0), vz.VZ_ERR_SHAPE),
                                              (dict(S=40000), vz.VZ_ERR_SHAPE), (dict(total=0), vz.VZ_ERR_SHAPE)])
def test_decode_q4_ragged_rejects(kw, code):
    a = dict(COMMON, b=FAKE, cap=FAKE, len=FAKE, next=FAKE, total=64, S=2, gamma=0.95, scale=0.0, L=2, Hq=32, Hkv=4,
             d=128, dtype=vz.VZ_BF16, status=None, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    assert vz.lib().voxzip_decode_attend_score_q4_ragged(*a.values(), None) == code


EVICT = [(dict(s=None), vz.VZ_ERR_INVALID), (dict(vc=None), vz.VZ_ERR_INVALID), (dict(kc=OFF8), vz.VZ_ERR_INVALID),
         (dict(ks=ODD), vz.VZ_ERR_INVALID), (dict(sink=-1), vz.VZ_ERR_INVALID), (dict(d=32), vz.VZ_ERR_UNSUPPORTED),
         (dict(ws=None), vz.VZ_ERR_WORKSPACE), (dict(ws_bytes=8), vz.VZ_ERR_WORKSPACE)]


@pytest.mark.parametrize("kw,code", EVICT + [(dict(budget=0), vz.VZ_ERR_INVALID), (dict(next_pos=99), vz.VZ_ERR_INVALID),
                                             (dict(len=129), vz.VZ_ERR_CAPACITY)])
def test_evict_q4_rejects(kw, code):
    n = ctypes.c_int32(-7)
    a = dict(kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, s=FAKE, p=FAKE, len=100, budget=50, sink=4, recent=-1, next_pos=100,
             kept=None, new=ctypes.byref(n), L=2, Hkv=4, d=128, cap=128, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    assert vz.lib().voxzip_evict_compact_q4(*a.values(), None) == code


def test_evict_q4_without_work_returns_length_and_queues_nothing():
    n = ctypes.c_int32(-7)
    assert vz.lib().voxzip_evict_compact_q4(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 40, 50, 4, -1, 100, None,
                                            ctypes.byref(n), 2, 4, 128, 128, None, 0, None) == vz.VZ_OK
    assert n.value == 40


@pytest.mark.parametrize("kw,code", EVICT + [(dict(b=None), vz.VZ_ERR_INVALID), (dict(S=0), vz.VZ_ERR_SHAPE),
                                             (dict(new=FAKE), vz.VZ_ERR_INVALID)])  # new_len_out on len
def test_evict_q4_ragged_rejects(kw, code):
    a = dict(kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, s=FAKE, p=FAKE, b=FAKE, cap=FAKE, len=FAKE, budget=FAKE, next=FAKE,
             total=64, S=2, sink=4, recent=-1, kept=None, new=None, status=None, L=2, Hkv=4, d=128, ws=FAKE,
             ws_bytes=1 << 30)
    a.update(kw)
    assert vz.lib().voxzip_evict_compact_q4_ragged(*a.values(), None) == code


def test_planes_of_more_than_2_26_slots_are_refused():
    n, big, L = ctypes.c_int32(-7), (1 << 26) + 1, vz.lib()
    ten, six = (FAKE,) * 10, (FAKE,) * 6
    tail = (1, 4, 2, 128, big, vz.VZ_BF16, FAKE, 1 << 40, None)
    assert L.voxzip_decode_attend_score_q4(*ten, 10, 10, 0.9, 0.0, *tail) == vz.VZ_ERR_SHAPE
    assert L.voxzip_decode_evict_q4(*ten, 10, 10, 0.9, 0.0, 10, 4, -1, None, ctypes.byref(n), *tail) == vz.VZ_ERR_SHAPE
    assert L.voxzip_evict_compact_q4(*six, 10, 5, 0, 0, 10, None, ctypes.byref(n), 1, 2, 128, big, FAKE, 1 << 40,
                                     None) == vz.VZ_ERR_SHAPE
    assert L.voxzip_fuse_spans_q4(FAKE, FAKE, 8, FAKE, 4, None, None, *six, 1, 2, 128, big, vz.VZ_BF16,
                                  None) == vz.VZ_ERR_SHAPE
    assert n.value == -7


def test_workspace_sizes_grow_with_the_cache():
    size = vz.voxzip_workspace_bytes
    for op in (vz.VZ_OP_DECODE_Q4, vz.VZ_OP_DECODE_EVICT_Q4):
        assert size(op, 0, 32, 4, 128, 64) == 0 and size(op, 2, 0, 4, 128, 64) == 0
        last = 0
        for cap in (1, 32, 33, 500, 8194, 70000, 1 << 20):
            assert size(op, 48, 32, 4, 128, cap) >= last > -1
            last = size(op, 48, 32, 4, 128, cap)
    assert vz.voxzip_workspace_bytes_ragged(vz.VZ_OP_DECODE_Q4, 2, 32, 4, 128, 500, 3) > 0
    assert vz.voxzip_workspace_bytes_ragged(vz.VZ_OP_DECODE_EVICT_Q4, 2, 32, 4, 128, 500, 3) == 0


def test_binding_checks_shapes_types_and_devices():
    import torch
    c = vz.q4_cache(2, 4, 10, 128, device="cpu")
    assert [tuple(x.shape) for x in c] == [(2, 4, 10, 64), (2, 4, 10, 4)] * 2
    q, kn = torch.zeros(2, 8, 128), torch.zeros(2, 4, 128)
    s, p = torch.zeros(2, 10), torch.zeros(2, 10, dtype=torch.int32)
    step = lambda q=q, c=c, out=q: vz.voxzip_decode_attend_score_q4(q, kn, kn, *c, s, p, out, 3, 3, 0.9)
    with pytest.raises(ValueError, match="GPU"):
        step()
    with pytest.raises(ValueError, match="v_scales"):
        step(c=c[:3] + (c[3][..., :2],))
    with pytest.raises(TypeError, match="k_codes"):
        step(c=(c[0].int(),) + c[1:])
    with pytest.raises(ValueError, match="head size"):
        step(q=torch.zeros(2, 8, 96))
    with pytest.raises(ValueError, match="out"):
        step(out=torch.zeros(2, 4, 128))
    with pytest.raises(ValueError, match="scales"):
        vz.voxzip_unpack_q4(c[0], c[0], torch.zeros(2, 4, 10, 128))
