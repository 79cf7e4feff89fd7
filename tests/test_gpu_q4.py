"""GPU parity of the 4-bit cache's entry points: rows in and out bit for bit
against the format's definition, decode steps against the float64 oracle on the
values that the cache holds, eviction against the full-precision eviction of
the same values."""


import numpy as np
import pytest

import oracle
import q4ref
import synth
from vzt import RTOL, check_close, check_rel, from_dev, to_dev, widen

pytestmark = pytest.mark.gpu

# Scores are float32 throughout in both element types, as on the general path:
# each p carries the rounding of its logit (d products of exact factors, |s| d
# 2^-24 at worst, a few 2^-24 in practice), one of exp2 and one of 1 / Z.
SCORE_RTOL = RTOL[synth.DT_F32]
BF16, F32 = synth.DT_BF16, synth.DT_F32
NAMES = ("k_codes", "k_scales", "v_codes", "v_scales")


def vz():
    import paper_2608_08569_amd as m
    return m


def torch():
    import torch as t
    return t


def store(x, dtype):
    return synth.as_storage(np.asarray(x, dtype=np.float32), dtype)


def i32(x):
    return torch().tensor(x, dtype=torch().int32, device="cuda")


def i64(x):
    return torch().tensor(x, dtype=torch().int64, device="cuda")


class Case:
    """A 4-bit cache with its score and position planes, on host and device."""

    def __init__(self, seed, L, Hq, Hkv, d, slots, dtype, spread=1.0):
        self.rng = np.random.default_rng(seed)
        self.L, self.Hq, self.Hkv, self.d, self.slots, self.dtype = L, Hq, Hkv, d, slots, dtype
        g = lambda *s: self.rng.standard_normal(s)
        ch = np.exp(spread * g(L, Hkv, 1, d) * 0.5)
        self.kc, self.ks = q4ref.quantise(g(L, Hkv, slots, d) * ch)
        self.vc, self.vs = q4ref.quantise(g(L, Hkv, slots, d) * ch)
        self.s = np.exp(2 * g(L, slots)).astype(np.float32) * np.float32(0.01)
        self.p = np.stack([self.rng.permutation(slots).astype(np.int32) for _ in range(L)])

    def rows(self, *lead):
        g = lambda h: store(self.rng.standard_normal((*lead, self.L, h, self.d)), self.dtype)
        return g(self.Hq), g(self.Hkv), g(self.Hkv)

    def hide(self, free):
        """Slots that hold nothing: blocks that read as NaN."""
        for c, s in ((self.kc, self.ks), (self.vc, self.vs)):
            c[:, :, free], s[:, :, free] = 0x77, 255

    def dev(self):
        return [to_dev(x) for x in (self.kc, self.ks, self.vc, self.vs)], to_dev(self.s), to_dev(self.p)

    def expect(self, q, kn, vn, base, length, next_pos, gamma, scale=0.0):
        """The oracle's step on the values held at slots base .. (q, kn, vn [L][..][d])."""
        f = lambda x: widen(x, self.dtype)
        at = slice(base, base + length + 1)
        K, V = (q4ref.values(c[:, :, at], s[:, :, at]) for c, s in ((self.kc, self.ks), (self.vc, self.vs)))
        K[:, :, length], V[:, :, length] = 0, 0  # (the step's own slot)
        new = [q4ref.quantise(f(x)) for x in (kn, vn)]
        f32 = lambda x: np.ascontiguousarray(x, dtype=np.float32)
        o, s, p, _ = oracle.decode_step(f32(f(q)), f32(q4ref.values(*new[0])), f32(q4ref.values(*new[1])), f32(K), f32(V),
                                        self.s[:, at].astype(np.float64), np.ascontiguousarray(self.p[:, at]), length,
                                        next_pos, gamma, F32, sm_scale=scale)
        return o, s, p, new

    def check_cache(self, cache, new, slots):
        """The appended rows bit for bit, every other row untouched. new: per sequence; slots: theirs."""
        for x, name, ref in zip(cache, NAMES, (self.kc, self.ks, self.vc, self.vs)):
            ref = ref.copy()
            for n, at in zip(new, slots):
                ref[:, :, at] = n["kv".index(name[0])]["cs".index(name[2])]
            assert np.array_equal(from_dev(x), ref), name


# ---- rows in and out ----

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,rows", [(64, 1), (64, 77), (128, 1), (128, 501)])
def test_unpack_every_code_and_scale(dtype, d, rows):
    rng = np.random.default_rng(rows)
    codes = rng.integers(0, 256, (rows, d // 2)).astype(np.uint8)
    scales = rng.choice(np.r_[2:253, 255], (rows, d // 32)).astype(np.uint8)
    codes.reshape(-1)[: 32] = np.arange(16).repeat(2) * 17
    out = torch().zeros(rows, d, dtype=torch().bfloat16 if dtype == BF16 else torch().float32, device="cuda")
    vz().voxzip_unpack_q4(to_dev(codes), to_dev(scales), out)
    assert np.array_equal(widen(from_dev(out), dtype), q4ref.values(codes, scales), equal_nan=True)
    out.fill_(3)
    vz().voxzip_unpack_q4(to_dev(codes), torch().zeros_like(to_dev(scales)) * 0, out)  # scale byte 0, codes 0
    vz().voxzip_unpack_q4(to_dev(codes * 0), to_dev(scales * 0), out)
    assert not from_dev(out).any()


def hard_rows(rng, T, d):
    """Values on and near the codes' borders, of every size, zeros, and blocks of one large value."""
    x = rng.standard_normal((T, d)) * 2.0 ** rng.integers(-30, 30, (T, 1))
    x[: T // 4] = rng.integers(-28, 29, (T // 4, d)) / 4
    x[T // 4: T // 2] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, -7, -5, 0, -0.0], (T // 2 - T // 4, d))
    x[T // 2, : 32] = 0
    x[T // 2 + 1, :] = 0
    x[T // 2 + 1, 5] = 3e38
    x[T // 2 + 2, :] = 1e-39
    x[-1, :] = 1e-37
    return x


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,L,H,T,anchor", [(128, 2, 3, 700, False), (64, 1, 1, 1, False), (64, 2, 2, 999, True),
                                            (128, 1, 5, 333, True), (64, 3, 1, 64, False)])
def test_fused_rows_bit_for_bit(dtype, d, L, H, T, anchor):
    rng = np.random.default_rng(T + d)
    k, v = (store(np.stack([hard_rows(rng, T, d) if T > 8 else rng.standard_normal((T, d)) for _ in range(L * H)])
                  .reshape(L, H, T, d), dtype) for _ in range(2))
    cuts = np.sort(rng.choice(T - 1, size=min(T - 1, T // 3), replace=False) + 1) if T > 1 else []
    off = np.concatenate([[0], cuts, [T]]).astype(np.int32)
    n, cap = len(off) - 1, len(off) + 4
    ak, av = (store(rng.integers(-8, 9, (L, H, n, d)) / 4, dtype) if anchor else None for _ in range(2))
    f = lambda x: None if x is None else widen(x, dtype)
    cache = vz().q4_cache(L, H, cap, d)
    for x in cache:
        x.fill_(0xA5)
    s, p = torch().full((L, cap), 9.0, device="cuda"), torch().full((L, cap), -9, dtype=torch().int32, device="cuda")
    on = lambda x: None if x is None else to_dev(x)
    vz().voxzip_fuse_spans_q4(to_dev(k), to_dev(v), to_dev(off), *cache, s, p, anchor_k=on(ak), anchor_v=on(av))
    want = q4ref.span_means(f(k), off, f(ak)) + q4ref.span_means(f(v), off, f(av))
    for x, ref, name in zip(cache, want, NAMES):
        got = from_dev(x)
        assert np.array_equal(got[:, :, :n], ref), name
        assert (got[:, :, n:] == 0xA5).all(), name  # the free slots stay as they were
    assert np.array_equal(from_dev(p)[:, :n], np.tile(np.arange(n), (L, 1))) and (from_dev(p)[:, n:] == -9).all()
    assert not from_dev(s)[:, :n].any() and (from_dev(s)[:, n:] == 9).all()


def test_a_plane_of_more_than_4_gib_is_fused():
    T, d, step = (1 << 24) + 77, 128, 64
    x = torch().empty(1, 1, T, d, dtype=torch().bfloat16, device="cuda").fill_(1.0)
    rng = np.random.default_rng(5)
    tail = store(hard_rows(rng, 4096, d), BF16)
    x[0, 0, T - 4096:] = to_dev(tail)
    off = np.concatenate([np.arange(0, T - 4096, step), np.arange(T - 4096, T, 3), [T]]).astype(np.int32)
    n, m = len(off) - 1, len(np.arange(T - 4096, T, 3))
    cache = vz().q4_cache(1, 1, n, d)
    s, p = torch().empty(1, n, device="cuda"), torch().empty(1, n, dtype=torch().int32, device="cuda")
    vz().voxzip_fuse_spans_q4(x, x, to_dev(off), *cache, s, p)
    codes, scales = q4ref.span_means(widen(tail, BF16)[None, None], off[n - m:] - off[n - m])
    for got, want in zip(cache, (codes, scales) * 2):
        assert np.array_equal(from_dev(got[:, :, n - m:]), want)
        assert (got[:, :, :n - m] == (0x66 if got.shape[-1] == d // 2 else 127 - 2)).all()  # 1 = 4 * 2^-2


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_blocks_that_are_not_finite_read_as_nan(dtype):
    x = np.ones((1, 1, 4, 128), dtype=np.float32)
    x[0, 0, 0, 3], x[0, 0, 1, 40], x[0, 0, 2, 127] = np.nan, np.inf, -np.inf
    x = store(x, dtype)
    cache, s, p = vz().q4_cache(1, 1, 4, 128), torch().zeros(1, 4, device="cuda"), i32([[0] * 4])
    vz().voxzip_fuse_spans_q4(to_dev(x), to_dev(x), i32(range(5)), *cache, s, p)
    bad = np.zeros((4, 4), dtype=bool)
    bad[0, 0] = bad[1, 1] = bad[2, 3] = True
    assert np.array_equal(from_dev(cache[1])[0, 0] == 255, bad) and np.array_equal(from_dev(cache[3])[0, 0] == 255, bad)
    out = torch().zeros(1, 1, 4, 128, device="cuda")
    vz().voxzip_unpack_q4(cache[0], cache[1], out)
    got = from_dev(out)[0, 0].reshape(4, 4, 32)
    assert np.isnan(got[bad]).all() and (got[~bad] == 1).all()
    # and as the new row of a decode step
    kn = to_dev(x[:, :, 1].copy())
    q = torch().ones(1, 1, 128, dtype=kn.dtype, device="cuda")
    vz().voxzip_decode_attend_score_q4(q, kn, kn, *cache, s, p, torch().zeros_like(q), 3, 3, 0.9,
                                       workspace=vz().workspace(vz().VZ_OP_DECODE_Q4, 1, 1, 1, 128, 4))
    assert from_dev(cache[1])[0, 0, 3].tolist() == from_dev(cache[3])[0, 0, 3].tolist() == [127 - 2, 255, 125, 125]


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_ragged_fusion_is_the_single_calls(dtype, d):
    rng = np.random.default_rng(5)
    L, H, T, n = 2, 2, [40, 9, 1, 70, 30], [13, 9, 1, 70, 30]
    in_base, total_in, base, total = [3, 50, 60, 62, 135], 170, [2, 20, 30, 40, 115], 160
    caps = [14, 9, 1, 69, 0]  # the fourth has no room for its spans, the fifth is idle
    k, v = (store(rng.standard_normal((L, H, total_in, d)), dtype) for _ in range(2))
    ak, av = (store(rng.standard_normal((L, H, total, d)), dtype) for _ in range(2))
    offs = [np.concatenate([[0], np.sort(rng.choice(t - 1, m - 1, replace=False) + 1), [t]]).astype(np.int32)
            for t, m in zip(T, n)]
    off_base = np.concatenate([[0], np.cumsum([len(o) for o in offs])[:-1]])
    cache = vz().q4_cache(L, H, total, d)
    for x in cache:
        x.fill_(0x5A)
    s, p, st = torch().full((L, total), 7.0, device="cuda"), i32([[-7] * total] * L), i32([99] * 5)
    K, V, AK, AV = (to_dev(x) for x in (k, v, ak, av))
    vz().voxzip_fuse_spans_q4_ragged(K, V, i64(in_base), i32(T), i32(np.concatenate(offs).tolist()),
                                     i64(off_base.tolist()), i32(n), max(n), *cache, s, p, i64(base), i32(caps),
                                     status=st, anchor_k=AK, anchor_v=AV)
    m = vz()
    assert from_dev(st).tolist() == [m.VZ_OK, m.VZ_OK, m.VZ_OK, m.VZ_ERR_CAPACITY, m.VZ_IDLE]
    free = np.ones(total, dtype=bool)
    for i in range(3):
        one = m.q4_cache(L, H, n[i], d)
        s1, p1 = torch().ones(L, n[i], device="cuda"), i32([[5] * n[i]] * L)
        rows, slots = slice(in_base[i], in_base[i] + T[i]), slice(base[i], base[i] + n[i])
        part = lambda x, at: x[:, :, at].contiguous()
        m.voxzip_fuse_spans_q4(part(K, rows), part(V, rows), to_dev(offs[i]), *one, s1, p1, anchor_k=part(AK, slots),
                               anchor_v=part(AV, slots))
        for x, y in zip(cache, one):
            assert torch().equal(x[:, :, slots], y)
        assert torch().equal(p[:, slots], p1) and torch().equal(s[:, slots], s1)
        free[slots] = False
    for x in cache:
        assert (from_dev(x)[:, :, free] == 0x5A).all()
    assert (from_dev(s)[:, free] == 7).all() and (from_dev(p)[:, free] == -7).all()


@pytest.mark.parametrize("n,dtype,d,H", [(5, F32, 64, 2), (63, BF16, 64, 2), (64, BF16, 128, 6), (65, F32, 64, 5),
                                         (200, BF16, 64, 2), (200, F32, 128, 3)])
def test_ragged_fusion_of_many_sequences(n, dtype, d, H):
    """Lengths from one row to thousands, idle slots and refused sequences between them."""
    m, t, L = vz(), torch(), 1
    rng = np.random.default_rng(n)
    T = np.where(rng.random(n) < 0.1, 2500, rng.integers(1, 60, n))
    T[-1] = 3000
    spans = np.maximum(1, T // rng.integers(1, 5, n))
    cap = spans + rng.integers(0, 3, n)
    idle, wrong = rng.random(n) < 0.2, rng.random(n) < 0.1
    idle[-1] = wrong[-1] = False
    offs = [np.concatenate([[0], np.sort(rng.choice(a - 1, b - 1, replace=False) + 1), [a]]) for a, b in zip(T, spans)]
    ahead = lambda x: np.concatenate([[0], np.cumsum(x)[:-1]])
    base, in_base, off_base = ahead(cap), ahead(T), ahead(spans + 1)
    K, V = (store(rng.standard_normal((L, H, T.sum(), d)), dtype) for _ in "kv")
    total = int(cap.sum())
    cache = m.q4_cache(L, H, total, d)
    for x in cache:
        x.fill_(0x5A)
    s, p = t.full((L, total), 7.0, device="cuda"), i32([[-7] * total] * L)
    st = i32([99] * n)
    m.voxzip_fuse_spans_q4_ragged(to_dev(K), to_dev(V), i64(in_base.tolist()), i32(T.tolist()),
                                  i32(np.concatenate(offs).tolist()), i64(off_base.tolist()),
                                  i32(np.where(wrong, T + 1, spans).tolist()), int(spans.max()), *cache, s, p,
                                  i64(base.tolist()), i32(np.where(idle, 0, cap).tolist()), status=st)
    assert from_dev(st).tolist() == [m.VZ_IDLE if i else m.VZ_ERR_SHAPE if w else m.VZ_OK for i, w in zip(idle, wrong)]
    free = np.ones(total, dtype=bool)
    got = [from_dev(x) for x in cache]
    for i in np.flatnonzero(~idle & ~wrong):
        at, rows = slice(base[i], base[i] + spans[i]), slice(in_base[i], in_base[i] + T[i])
        want = sum((q4ref.span_means(widen(x[:, :, rows], dtype), offs[i]) for x in (K, V)), ())
        for x, y, name in zip(got, want, NAMES):
            assert np.array_equal(x[:, :, at], y), (i, name)
        assert (from_dev(p)[:, at] == np.arange(spans[i])).all() and not from_dev(s)[:, at].any()
        free[at] = False
    for x in got:
        assert (x[:, :, free] == 0x5A).all()
    assert (from_dev(s)[:, free] == 7).all() and (from_dev(p)[:, free] == -7).all()


# ---- decode ----

SHAPES = [(BF16, 128, 32, 4), (F32, 128, 6, 3), (BF16, 64, 14, 2), (F32, 64, 4, 1), (BF16, 128, 16, 1),
          (F32, 128, 18, 2), (BF16, 64, 5, 5), (BF16, 128, 64, 8), (F32, 64, 9, 1)]
LENGTHS = [0, 1, 30, 31, 32, 127, 255, 700]


def run_single(c, length, next_pos, gamma, L, scale=0.0, large_logits=False):
    q, kn, vn = c.rows()
    more = 0.0
    if large_logits:
        # A logit s is added up in float32 over d / 32 products of 32 channels and scaled: d / 32 + 1 roundings of
        # at most 2^-24 |s| each, by which p = exp(s - max) / Z is off relative to itself, once for its own s and
        # once for those in Z (the max cancels).
        K = q4ref.values(c.kc, c.ks).reshape(c.L, c.Hkv, 1, c.slots, c.d)
        Q = widen(q, c.dtype).reshape(c.L, c.Hkv, -1, 1, c.d)
        more = 2 * (c.d // 32 + 1) * 2.0 ** -24 * (scale or c.d ** -0.5) * np.abs((Q * K).sum(-1)).max()
    c.hide(slice(length, None))
    cache, s, p = c.dev()
    out = torch().full((L, c.Hq, c.d), 5.0, dtype=to_dev(q).dtype, device="cuda")
    ws = vz().workspace(vz().VZ_OP_DECODE_Q4, L, c.Hq, c.Hkv, c.d, c.slots)
    ws.fill_(0xFF)  # the workspace needs no initialisation (here: NaNs)
    vz().voxzip_decode_attend_score_q4(to_dev(q), to_dev(kn), to_dev(vn), *cache, s, p, out, length, next_pos, gamma,
                                       sm_scale=scale, workspace=ws)
    ref_o, ref_s, ref_p, new = c.expect(q, kn, vn, 0, length, next_pos, gamma, scale)
    check_close(widen(from_dev(out), c.dtype), ref_o, RTOL[c.dtype] + more, "output")
    check_rel(from_dev(s)[:, : length + 1], ref_s, SCORE_RTOL + more, "score")
    assert np.array_equal(from_dev(s)[:, length + 1:], c.s[:, length + 1:])
    assert np.array_equal(from_dev(p)[:, : length + 1], ref_p)
    assert np.array_equal(from_dev(p)[:, length + 1:], c.p[:, length + 1:])
    c.check_cache(cache, [new], [length])


@pytest.mark.parametrize("length", LENGTHS)
@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES)
def test_decode_against_oracle(dtype, d, Hq, Hkv, length):
    c = Case(length + d, 2, Hq, Hkv, d, length + 3, dtype)
    run_single(c, length, length + 9, 0.95, 2)


@pytest.mark.parametrize("dtype,d,Hq,Hkv,L,length", [
    (BF16, 128, 32, 4, 1, 8200), (BF16, 64, 14, 2, 1, 17000), (F32, 128, 8, 4, 1, 9001), (BF16, 128, 8, 8, 48, 600),
    (F32, 64, 2, 1, 300, 40), (BF16, 128, 4, 1, 70, 1023), (BF16, 128, 16, 2, 3, 1024)])
def test_decode_of_many_chunks_and_layers(dtype, d, Hq, Hkv, L, length):
    run_single(Case(3, L, Hq, Hkv, d, length + 1, dtype), length, length, 0.9, L)


@pytest.mark.parametrize("more", [-32, -1, 0, 1])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", SHAPES + [(BF16, 128, 16, 16), (F32, 128, 12, 12), (BF16, 64, 17, 17)])
def test_decode_around_whole_units_of_keys(dtype, d, Hq, Hkv, more):
    units = 140 // (Hkv * (1 if Hq // Hkv <= 8 else 2))
    length = 32 * units - 1 + more
    run_single(Case(length, 2, Hq, Hkv, d, length + 1, dtype), length, length, 0.95, 2)


@pytest.mark.parametrize("length", [0, 1, 31, 32, 63])
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 64)])
def test_short_caches_of_many_layers(dtype, d, length):
    run_single(Case(length, 257, 2, 1, d, length + 1, dtype), length, length, 0.95, 257)


@pytest.mark.parametrize("gamma,scale", [(0.0, 0.0), (1.0, 0.5), (0.5, 1e-3)])
def test_decode_decay_and_scale(gamma, scale):
    run_single(Case(8, 2, 8, 2, 128, 300, BF16), 290, 300, gamma, 2, scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_part_of_the_keys_far_below_the_rest(dtype):
    """Logits that underflow to a weight of 0 in whole chunks and at their ends."""
    c = Case(4, 2, 8, 2, 128, 400, dtype)
    big = np.zeros((2, 2, 400, 128))
    big[:, :, :, 7] = np.where(np.arange(400) % 100 < 64, -6.0, 6.0) * 2.0 ** 6
    c.kc, c.ks = q4ref.quantise(big + q4ref.values(c.kc, c.ks) * (np.arange(128) // 32 > 0))
    run_single(c, 390, 390, 0.9, 2, scale=1.0, large_logits=True)


@pytest.mark.parametrize("dtype,d,Hq,Hkv", [(BF16, 128, 8, 2), (F32, 64, 9, 1), (BF16, 64, 18, 2)])
def test_a_query_that_is_not_finite_is_its_heads_alone(dtype, d, Hq, Hkv):
    """Its outputs and its layer's scores are NaN; every other head's outputs keep their bits."""
    m, t, n = vz(), torch(), 150
    c = Case(7, 3, Hq, Hkv, d, n + 1, dtype)
    q, kn, vn = (to_dev(x) for x in c.rows())
    results = []
    for bad in (False, True):
        cache, s, p = c.dev()
        if bad:
            q[0, 1, 3], q[2, Hq - 1, d - 1] = float("inf"), float("nan")
        out = t.zeros_like(q)
        m.voxzip_decode_attend_score_q4(q, kn, vn, *cache, s, p, out, n, n, 0.9,
                                        workspace=m.workspace(m.VZ_OP_DECODE_Q4, 3, Hq, Hkv, d, n + 1))
        results.append((out, s, *cache))
    (o0, s0, *c0), (o1, s1, *c1) = results
    hit = t.zeros(3, Hq, dtype=t.bool, device="cuda")
    hit[0, 1] = hit[2, Hq - 1] = True
    assert o1[hit].isnan().all() and t.equal(o1[~hit], o0[~hit]) and not o0.isnan().any()
    assert s1[[0, 2]].isnan().all() and t.equal(s1[1], s0[1])
    assert all(t.equal(x, y) for x, y in zip(c0, c1))


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 128), (F32, 64)])
def test_inputs_and_outputs_at_any_element_alignment(dtype, d):
    m, t, L, Hq, Hkv, n = vz(), torch(), 2, 6, 2, 130
    c = Case(17, L, Hq, Hkv, d, n + 1, dtype)
    rows = [to_dev(x) for x in c.rows()]
    k, v = (to_dev(store(c.rng.standard_normal((L, Hkv, 400, d)), dtype)) for _ in "kv")
    ak, av = (to_dev(store(c.rng.standard_normal((L, Hkv, n, d)), dtype)) for _ in "kv")
    off = i32(sorted(c.rng.choice(399, n - 1, replace=False) + 1))
    off = t.cat([i32([0]), off, i32([400])])

    def odd(x):
        """The same values one element further on."""
        y = t.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
        y.copy_(x)
        return y

    results = []
    for move in (lambda x: x, odd):
        cache, s, p = m.q4_cache(L, Hkv, n + 1, d), t.zeros(L, n + 1, device="cuda"), i32([[0] * (n + 1)] * L)
        m.voxzip_fuse_spans_q4(move(k), move(v), off, *cache, s, p, anchor_k=move(ak), anchor_v=move(av))
        out = move(t.zeros_like(rows[0]))
        m.voxzip_decode_attend_score_q4(*(move(x) for x in rows), *cache, s, p, out, n, n, 0.9,
                                        workspace=m.workspace(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, n + 1))
        results.append((*cache, s, p, out))
    for x, y in zip(*results):
        assert t.equal(x, y)


@pytest.mark.parametrize("dtype,d,Hq,Hkv,L", [(BF16, 128, 32, 4, 2), (F32, 64, 4, 1, 3), (BF16, 64, 18, 2, 1),
                                              (F32, 128, 10, 5, 1)])
def test_ragged_decode_against_oracle(dtype, d, Hq, Hkv, L):
    m = vz()
    lens, caps = [0, 40, 5, 700, 31, 7, 3, 2000], [1, 41, 0, 705, 40, 7, 9, 2001]  # 2: idle, 5: full
    base = (np.cumsum([0] + [c + 3 for c in caps])[:-1] + 1).tolist()
    nxt = [n + 4 for n in lens]
    nxt[6] = -1  # refused
    total = base[-1] + caps[-1] + 2
    c = Case(d + Hq, L, Hq, Hkv, d, total, dtype)
    free = np.ones(total, dtype=bool)
    for b, n in zip(base, lens):
        free[b: b + n] = False
    c.hide(free)
    q, kn, vn = c.rows(len(lens))
    cache, s, p = c.dev()
    out = torch().full(q.shape, 5.0, dtype=to_dev(q).dtype, device="cuda")
    st, ws = i32([99] * 8), m.workspace_ragged(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, total, 8)
    ws.fill_(0xFF)
    m.voxzip_decode_attend_score_q4_ragged(to_dev(q), to_dev(kn), to_dev(vn), *cache, s, p, out, i64(base), i32(caps),
                                           i32(lens), i32(nxt), 0.95, status=st, workspace=ws)
    ok = [0, 1, 3, 4, 7]
    assert from_dev(st).tolist() == [m.VZ_OK, m.VZ_OK, m.VZ_IDLE, m.VZ_OK, m.VZ_OK, m.VZ_ERR_CAPACITY,
                                     m.VZ_ERR_INVALID, m.VZ_OK]
    got_s, got_p, news = from_dev(s), from_dev(p), []
    for i in range(8):
        if i not in ok:
            assert (from_dev(out)[i] == from_dev(torch().full((1,), 5.0, dtype=out.dtype))[0]).all()
            continue
        at = slice(base[i], base[i] + lens[i] + 1)
        ref_o, ref_s, ref_p, new = c.expect(q[i], kn[i], vn[i], base[i], lens[i], nxt[i], 0.95)
        check_close(widen(from_dev(out)[i], dtype), ref_o, RTOL[dtype], f"output {i}")
        check_rel(got_s[:, at], ref_s, SCORE_RTOL, f"score {i}")
        assert np.array_equal(got_p[:, at], ref_p)
        news.append(new)
        free[base[i] + lens[i]] = False
    c.check_cache(cache, news, [base[i] + lens[i] for i in ok])
    assert np.array_equal(got_s[:, free], c.s[:, free]) and np.array_equal(got_p[:, free], c.p[:, free])


def test_ragged_decode_of_many_short_sequences():
    m, n, L, Hq, Hkv, d = vz(), 333, 1, 4, 2, 64
    lens = [i * 7 % 41 for i in range(n)]
    base = np.cumsum([0] + [x + 1 for x in lens])
    total = int(base[-1])
    c = Case(2, L, Hq, Hkv, d, total, BF16)
    q, kn, vn = c.rows(n)
    cache, s, p = c.dev()
    out = torch().zeros(q.shape, dtype=torch().bfloat16, device="cuda")
    m.voxzip_decode_attend_score_q4_ragged(
        to_dev(q), to_dev(kn), to_dev(vn), *cache, s, p, out, i64(base[:-1].tolist()), i32([x + 1 for x in lens]),
        i32(lens), i32(lens), 0.9, workspace=m.workspace_ragged(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, total, n))
    for i in (0, 1, 63, 64, 65, 200, 331, 332):
        ref_o, ref_s, _, _ = c.expect(q[i], kn[i], vn[i], int(base[i]), lens[i], lens[i], 0.9)
        check_close(widen(from_dev(out)[i], BF16), ref_o, RTOL[BF16], f"output {i}")
        check_rel(from_dev(s)[:, base[i]: base[i + 1]], ref_s, SCORE_RTOL, f"score {i}")


# ---- eviction ----

def evicted(c, length, budget, next_pos, kept=True, n_sink=4, n_recent=-1):
    """The 4-bit eviction beside the full-precision one of the same values."""
    m, t = vz(), torch()
    cache, s, p = c.dev()
    full, s2, p2 = [t.zeros(c.L, c.Hkv, c.slots, c.d, dtype=t.bfloat16, device="cuda") for _ in "kv"], s.clone(), p.clone()
    unpack = lambda to: [m.voxzip_unpack_q4(cache[2 * i], cache[2 * i + 1], to[i]) for i in (0, 1)]
    unpack(full)
    ws = m.workspace(m.VZ_OP_EVICT, c.L, c.Hq, c.Hkv, c.d, c.slots)
    ka, kb = (t.full((c.L, budget), -1, dtype=t.int32, device="cuda") if kept else None for _ in range(2))
    n2 = m.voxzip_evict_compact(*full, s2, p2, length, budget, next_pos, n_sink, n_recent, kept_pos_out=kb, workspace=ws)
    ws.fill_(0xFF)
    n1 = m.voxzip_evict_compact_q4(*cache, s, p, length, budget, next_pos, n_sink, n_recent, kept_pos_out=ka, workspace=ws)
    assert n1 == n2 == min(length, budget)
    mine = [t.zeros_like(x) for x in full]
    unpack(mine)
    for x, y in zip(mine + [s, p], full + [s2, p2]):
        assert t.equal(x, y)
    if kept:
        assert t.equal(ka, kb)


@pytest.mark.parametrize("d,Hkv,L,length,budget", [
    (128, 4, 2, 129, 128), (64, 2, 3, 700, 695), (128, 1, 1, 3000, 2000), (64, 5, 2, 900, 300), (128, 2, 1, 17000, 16999),
    (128, 2, 1, 17000, 4000), (64, 1, 2, 64, 64), (128, 3, 1, 40, 100)])
def test_evict_is_the_full_precision_eviction(d, Hkv, L, length, budget):
    c = Case(length, L, Hkv, Hkv, d, length + 2, BF16)
    c.s[:, ::3] = 0.25  # equal scores: the smaller position stays
    evicted(c, length, budget, length + 2)
    evicted(c, length, budget, length + 2, kept=False, n_sink=0, n_recent=3)


@pytest.mark.parametrize("d", [64, 128])
def test_ragged_evict_is_the_single_calls(d):
    m, t, L, Hkv = vz(), torch(), 2, 3
    lens, budgets, caps = [300, 50, 10, 900, 20], [200, 60, 5, 100, 0], [310, 50, 0, 900, 20]
    base = [2, 330, 400, 420, 1330]
    total = 1360
    c = Case(d, L, Hkv, Hkv, d, total, BF16)
    pos = c.p.copy()
    for l in range(L):
        for b, n in zip(base, lens):
            pos[l, b: b + n] = c.rng.permutation(n + 3)[:n]
    c.p = pos
    cache, s, p = c.dev()
    nxt = [n + 3 for n in lens]
    kept, new_len, st = t.full((L, total), -1, dtype=t.int32, device="cuda"), i32([99] * 5), i32([99] * 5)
    ws = m.workspace_ragged(m.VZ_OP_EVICT, L, Hkv, Hkv, d, total, 5)
    ws.fill_(0xFF)
    m.voxzip_evict_compact_q4_ragged(*cache, s, p, i64(base), i32(caps), i32(lens), i32(budgets), i32(nxt),
                                     kept_pos_out=kept, new_len_out=new_len, status=st, workspace=ws)
    assert from_dev(st).tolist() == [m.VZ_OK, m.VZ_OK, m.VZ_IDLE, m.VZ_OK, m.VZ_ERR_INVALID]
    assert from_dev(new_len).tolist() == [200, 50, 10, 100, 20]
    ref, rs, rp = c.dev()
    for i in (0, 1, 3):
        at = slice(base[i], base[i] + caps[i])
        one = [x[:, :, at].contiguous() for x in ref]
        s1, p1 = rs[:, at].contiguous(), rp[:, at].contiguous()
        k1 = t.zeros(L, budgets[i], dtype=t.int32, device="cuda")
        n = m.voxzip_evict_compact_q4(*one, s1, p1, lens[i], budgets[i], nxt[i], kept_pos_out=k1,
                                      workspace=m.workspace(m.VZ_OP_EVICT, L, Hkv, Hkv, d, caps[i]))
        for x, y in zip(ref, one):
            x[:, :, at] = y
        rs[:, at], rp[:, at] = s1, p1
        assert t.equal(kept[:, base[i]: base[i] + n], k1[:, :n])
    for x, y in zip(cache + [s, p], ref + [rs, rp]):
        assert t.equal(x, y)


# ---- together ----

STEPS = [(BF16, 128, 32, 4, 1, 1024, 1024), (F32, 64, 4, 1, 2, 128, 128), (BF16, 64, 14, 2, 3, 300, 200),
         (BF16, 128, 16, 1, 1, 50, 100), (F32, 128, 10, 5, 2, 700, 690), (BF16, 128, 8, 2, 40, 90, 90),
         (BF16, 128, 32, 4, 1, 1300, 1300), (F32, 64, 4, 1, 2, 4600, 4600), (BF16, 64, 18, 2, 3, 2400, 2400),
         (F32, 128, 10, 5, 2, 700, 700), (BF16, 64, 16, 16, 1, 200, 200), (BF16, 64, 2, 1, 257, 40, 40)]


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("dtype,d,Hq,Hkv,L,length,budget", STEPS)
def test_step_is_decode_then_evict(dtype, d, Hq, Hkv, L, length, budget, kept):
    m, t = vz(), torch()
    c = Case(length + L, L, Hq, Hkv, d, length + 2, dtype)
    q, kn, vn = (to_dev(x) for x in c.rows())
    nxt = length + 5
    a, sa, pa = c.dev()
    b, sb, pb = c.dev()
    oa, ob = (t.zeros_like(q) for _ in range(2))
    ka, kb = (t.full((L, budget), -1, dtype=t.int32, device="cuda") if kept else None for _ in range(2))
    m.voxzip_decode_attend_score_q4(q, kn, vn, *a, sa, pa, oa, length, nxt, 0.95,
                                    workspace=m.workspace(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, c.slots))
    na = m.voxzip_evict_compact_q4(*a, sa, pa, length + 1, budget, nxt + 1, kept_pos_out=ka,
                                   workspace=m.workspace(m.VZ_OP_EVICT, L, Hq, Hkv, d, c.slots))
    ws = m.workspace(m.VZ_OP_DECODE_EVICT_Q4, L, Hq, Hkv, d, c.slots)
    ws.fill_(0xFF)
    nb = m.voxzip_decode_evict_q4(q, kn, vn, *b, sb, pb, ob, length, nxt, 0.95, budget, kept_pos_out=kb, workspace=ws)
    assert na == nb == min(length + 1, budget)
    for x, y in zip(a + [sa, pa, oa], b + [sb, pb, ob]):
        assert t.equal(x, y)
    if kept:
        assert t.equal(ka, kb)


@pytest.mark.parametrize("budget,n_sink,n_recent", [
    (1, 0, 0), (2, 0, 1), (5, 4, 0), (5, 4, 1), (40, 0, 0), (40, 39, 1), (40, 40, 0), (40, 0, 40)])
@pytest.mark.parametrize("spread", [0, 1])
def test_step_with_few_or_no_slots_that_compete(budget, n_sink, n_recent, spread):
    """One slot over the budget, where sinks and recent positions protect most
    of the slots or all, and where the scores are equal."""
    m, t, L, Hq, Hkv, d = vz(), torch(), 2, 4, 2, 64
    c = Case(budget, L, Hq, Hkv, d, budget + 1, BF16)
    if not spread:
        c.s[:] = 0
    q, kn, vn = (to_dev(x) for x in c.rows())
    if not spread:
        q.zero_()  # every key weighs the same
    results = []
    for split in (True, False):
        cache, s, p = c.dev()
        out = t.zeros_like(q)
        if split:
            m.voxzip_decode_attend_score_q4(q, kn, vn, *cache, s, p, out, budget, budget + 2, 0.9,
                                            workspace=m.workspace(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, c.slots))
            m.voxzip_evict_compact_q4(*cache, s, p, budget + 1, budget, budget + 3, n_sink, n_recent,
                                      workspace=m.workspace(m.VZ_OP_EVICT, L, Hq, Hkv, d, c.slots))
        else:
            m.voxzip_decode_evict_q4(q, kn, vn, *cache, s, p, out, budget, budget + 2, 0.9, budget, n_sink, n_recent,
                                     workspace=m.workspace(m.VZ_OP_DECODE_EVICT_Q4, L, Hq, Hkv, d, c.slots))
        results.append([x[:, :, : budget] for x in cache] + [s[:, : budget], p[:, : budget], out])
    for x, y in zip(*results):
        assert t.equal(x, y)


def test_calls_on_two_streams_at_once():
    """Each call with a workspace of its own: the bits of the calls one after the other."""
    m, t, L, Hq, Hkv, d = vz(), torch(), 8, 16, 2, 128
    cases = [Case(i, L, Hq, Hkv, d, 2050, BF16) for i in range(2)]
    rows = [[to_dev(x) for x in c.rows()] for c in cases]
    streams = [t.cuda.Stream(), t.cuda.Stream()]
    results = []
    for together in (False, True):
        state = [c.dev() for c in cases]
        outs = [t.zeros_like(r[0]) for r in rows]
        ws = [m.workspace(m.VZ_OP_DECODE_EVICT_Q4, L, Hq, Hkv, d, 2050) for _ in cases]
        t.cuda.synchronize()
        for step in range(4):
            for i in range(2):
                cache, s, p = state[i]
                m.voxzip_decode_evict_q4(*rows[i], *cache, s, p, outs[i], 2049, 2055 + step, 0.9, 2049, workspace=ws[i],
                                         stream=streams[i if together else 0])
        t.cuda.synchronize()
        results.append([x for (cache, s, p), o in zip(state, outs) for x in (*cache, s, p, o)])
    for x, y in zip(*results):
        assert t.equal(x, y)


def test_a_request_from_prefill_to_eviction():
    """Fusion, decode steps past the budget and evictions in a row, each step
    checked against the oracle on the state before it; on a stream of its own."""
    m, t, L, Hq, Hkv, d, T, n, budget = vz(), torch(), 2, 14, 2, 64, 400, 150, 140
    rng = np.random.default_rng(12)
    k, v = (store(rng.standard_normal((L, Hkv, T, d)), BF16) for _ in range(2))
    off = np.concatenate([[0], np.sort(rng.choice(T - 1, n - 1, replace=False) + 1), [T]]).astype(np.int32)
    c = Case(1, L, Hq, Hkv, d, n + 4, BF16)
    cache, s, p = m.q4_cache(L, Hkv, n + 4, d), t.zeros(L, n + 4, device="cuda"), i32([[0] * (n + 4)] * L)
    ws_d = m.workspace(m.VZ_OP_DECODE_EVICT_Q4, L, Hq, Hkv, d, n + 4)
    ws_e = m.workspace(m.VZ_OP_EVICT, L, Hq, Hkv, d, n + 4)
    kd, vd, od, out = to_dev(k), to_dev(v), to_dev(off), t.zeros(L, Hq, d, dtype=t.bfloat16, device="cuda")
    stream = t.cuda.Stream()
    stream.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(stream):
        m.voxzip_fuse_spans_q4(kd, vd, od, *cache, s, p)
        length, nxt = n, n
        for step in range(6):
            stream.synchronize()
            c.kc, c.ks, c.vc, c.vs, c.s, c.p = (from_dev(x) for x in cache + (s, p))
            q, kn, vn = c.rows()
            ref_o, ref_s, ref_p, _ = c.expect(q, kn, vn, 0, length, nxt, 0.95)
            dq, dk, dv = (to_dev(x) for x in (q, kn, vn))
            if step < 3:  # to n + 3 slots, then down to the budget
                m.voxzip_decode_attend_score_q4(dq, dk, dv, *cache, s, p, out, length, nxt, 0.95, workspace=ws_d)
                length += 1
            else:
                length = m.voxzip_decode_evict_q4(dq, dk, dv, *cache, s, p, out, length, nxt, 0.95, budget, workspace=ws_d)
                assert length == budget
            nxt += 1
            stream.synchronize()
            check_close(widen(from_dev(out), BF16), ref_o, RTOL[BF16], f"output {step}")
            got = from_dev(s)
            if step < 3:
                check_rel(got[:, :length], ref_s, SCORE_RTOL, f"score {step}")
            else:  # what the step kept: each position's score is its own
                for l in range(L):
                    of = dict(zip(ref_p[l].tolist(), ref_s[l].tolist()))
                    pos = from_dev(p)[l, :length].tolist()
                    assert len(set(pos)) == length and nxt - 1 in pos and {0, 1, 2, 3} <= set(pos)
                    check_rel(got[l, :length], np.array([of[x] for x in pos]), SCORE_RTOL, f"score {step}")
        m.voxzip_evict_compact_q4(*cache, s, p, length, 40, nxt, workspace=ws_e)
    stream.synchronize()


def test_a_captured_step_replays():
    """Two captured graphs sharing a workspace, replayed in turn with eager work
    between, give the eager calls' bits."""
    m, t, L, Hq, Hkv, d, budget = vz(), torch(), 3, 8, 2, 128, 300
    c = Case(9, L, Hq, Hkv, d, budget + 2, BF16)
    q, kn, vn = (to_dev(x) for x in c.rows())
    ws = m.workspace(m.VZ_OP_DECODE_EVICT_Q4, L, Hq, Hkv, d, c.slots)
    states = [c.dev() for _ in range(4)]
    outs = [t.zeros_like(q) for _ in range(4)]

    def step(i):
        cache, s, p = states[i]
        m.voxzip_decode_evict_q4(q, kn, vn, *cache, s, p, outs[i], budget, budget + 7, 0.9, budget, workspace=ws)

    flat = lambda i: states[i][0] + [states[i][1], states[i][2], outs[i]]
    fresh = [x.clone() for x in flat(0)]
    step(2)  # the eager result (and the first use, outside capture)
    graphs = []
    for i in (0, 1):
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            step(i)
        graphs.append(g)
    for r in range(4):
        for i in (0, 1, 3):
            for x, y in zip(flat(i), fresh):
                x.copy_(y)
        graphs[r % 2].replay()
        step(3)
        graphs[1 - r % 2].replay()
        t.cuda.synchronize()
        for i in (0, 1, 3):
            for x, y in zip(flat(i), flat(2)):
                assert t.equal(x, y), (r, i)


def test_tensors_of_another_device_are_refused(monkeypatch):
    """Told on the host, with a card's number that is not the tensors'."""
    m, t, n = vz(), torch(), 1
    c = Case(1, 1, 2, 1, 64, 4, BF16)
    cache, s, p = c.dev()
    q, kn, _ = (to_dev(x) for x in c.rows())
    out, ln, base = t.zeros_like(q), i32([n]), i64([0])
    rows, off = t.zeros(1, 1, 4, 64, dtype=t.bfloat16, device="cuda"), i32([0, 2, 4])
    calls = [
        lambda: m.voxzip_fuse_spans_q4(rows, rows, off, *cache, s, p),
        lambda: m.voxzip_unpack_q4(cache[0], cache[1], rows),
        lambda: m.voxzip_decode_attend_score_q4(q, kn, kn, *cache, s, p, out, n, n, 0.9),
        lambda: m.voxzip_evict_compact_q4(*cache, s, p, 3, 2, 3),
        lambda: m.voxzip_decode_evict_q4(q, kn, kn, *cache, s, p, out, n, n, 0.9, 2),
        lambda: m.voxzip_fuse_spans_q4_ragged(rows, rows, base, ln, off, base, ln, 2, *cache, s, p, base, ln),
        lambda: m.voxzip_decode_attend_score_q4_ragged(q[None], kn[None], kn[None], *cache, s, p, out[None], base, ln,
                                                       ln, ln, 0.9),
        lambda: m.voxzip_evict_compact_q4_ragged(*cache, s, p, base, ln, ln, ln, ln)]
    before = [x.clone() for x in (*cache, s, p, out, rows)]
    monkeypatch.setattr(t.cuda, "current_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
    s, full = s.cpu(), s
    for call in calls[:1] + calls[2:]:
        with pytest.raises(ValueError, match="one device"):
            call()
    monkeypatch.undo()
    for x, y in zip((*cache, full, p, out, rows), before):
        assert t.equal(x, y)


def test_slots_beyond_four_gigabytes():
    """Codes whose byte offsets pass 2^32 in one plane set."""
    m, t, L, Hq, Hkv, d, cap, length = vz(), torch(), 3, 2, 2, 128, 12_000_000, 200
    cache = [t.zeros(L, Hkv, cap, n, dtype=t.uint8, device="cuda") for n in (64, 4, 64, 4)]
    s, p = t.zeros(L, cap, device="cuda"), t.zeros(L, cap, dtype=t.int32, device="cuda")
    c = Case(6, L, Hq, Hkv, d, length + 1, BF16)
    at = cap - length - 1  # the last slots of the planes, as one sequence of a batch
    for x, y in zip(cache, (c.kc, c.ks, c.vc, c.vs)):
        x[:, :, at:] = to_dev(y)
    s[:, at:], p[:, at:] = to_dev(c.s), to_dev(c.p)
    q, kn, vn = c.rows(1)
    out = t.zeros(1, L, Hq, d, dtype=t.bfloat16, device="cuda")
    ws = m.workspace_ragged(m.VZ_OP_DECODE_Q4, L, Hq, Hkv, d, cap, 1)
    m.voxzip_decode_attend_score_q4_ragged(to_dev(q), to_dev(kn), to_dev(vn), *cache, s, p, out, i64([at]),
                                           i32([length + 1]), i32([length]), i32([length]), 0.9, workspace=ws)
    ref_o, ref_s, _, _ = c.expect(q[0], kn[0], vn[0], 0, length, length, 0.9)
    check_close(widen(from_dev(out)[0], BF16), ref_o, RTOL[BF16], "output")
    check_rel(from_dev(s[:, at:]), ref_s, SCORE_RTOL, "score")
    m.voxzip_evict_compact_q4_ragged(*cache, s, p, i64([at]), i32([length + 1]), i32([length + 1]), i32([100]),
                                     i32([length + 1]), workspace=m.workspace_ragged(m.VZ_OP_EVICT, L, Hq, Hkv, d, cap, 1))
    assert (from_dev(s[:, at: at + 100]) > 0).all()
