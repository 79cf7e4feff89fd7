"""The decode loop over a 4-bit cache (``DecodeLoop(bits=4)``): each step of
each sequence matches the oracle on the state before it, also of a request that
joined in a freed slot; graph replays give the bits of eager steps, in the
all-layer and the per-layer mode, with the eviction schedule."""
import numpy as np
import pytest

import q4ref
import synth
from test_gpu_q4 import BF16, F32, SCORE_RTOL, Case, i32, i64, store, torch
from vzt import RTOL, check_close, check_rel, from_dev, to_dev, widen

pytestmark = pytest.mark.gpu

T_IN, BUDGETS, INTERVAL, STEPS, GAMMA = [900, 2500, 120], [180, 500, 24], 2, 7, 0.95


def _spans(rng, T):
    return np.concatenate([[0], np.sort(rng.choice(T - 1, T // 4 - 1, replace=False) + 1), [T]]).astype(np.int32)


def _loop(shape, seed=21):
    """A loop whose sequences hold their fused prefills, and its host side."""
    from paper_2608_08569_amd.loop import DecodeLoop
    dtype, d, Hq, Hkv, L = shape
    rng = np.random.default_rng(seed)
    offs = [_spans(rng, T) for T in T_IN]
    n = [len(o) - 1 for o in offs]
    caps = np.maximum(n, BUDGETS) + INTERVAL + 2
    lp = DecodeLoop(L, Hq, Hkv, d, caps, BUDGETS, GAMMA, interval=INTERVAL, bits=4,
                    dtype=torch().float32 if dtype == F32 else torch().bfloat16)
    kv = [store(rng.standard_normal((L, Hkv, sum(T_IN), d)), dtype) for _ in "kv"]
    start = np.concatenate([[0], np.cumsum(T_IN)[:-1]])
    lp.fuse(*(to_dev(x) for x in kv), i64(start.tolist()), i32(T_IN), to_dev(np.concatenate(offs)),
            i64(np.concatenate([[0], np.cumsum([x + 1 for x in n])[:-1]]).tolist()), i32(n), max(n))
    assert from_dev(lp.status).tolist() == [0, 0, 0]
    c = Case(seed, L, Hq, Hkv, d, lp.total, dtype)
    for s, (t0, T, o) in enumerate(zip(start, T_IN, offs)):
        b = int(lp.seq_base[s])
        for x, planes in zip(kv, (lp.planes[:2], lp.planes[2:])):
            want = q4ref.span_means(widen(x[:, :, t0: t0 + T], dtype), o)
            for got, ref in zip(planes, want):
                assert np.array_equal(from_dev(got[:, :, b: b + n[s]]), ref)
    return lp, c


def _state(lp):
    torch().cuda.synchronize()
    return [from_dev(x) for x in (*lp.planes, lp.score, lp.pos, lp.length, lp.next_pos, lp.status)]


def _check_step(lp, c, before, q, kn, vn, out):
    """Outputs of every active sequence, and the scores and rows that its step left in place."""
    c.kc, c.ks, c.vc, c.vs, c.s, c.p, lens, nxts, _ = before
    after = _state(lp)
    for s in np.flatnonzero(lp.active):
        b, n, nxt = int(lp.seq_base[s]), int(lens[s]), int(nxts[s])
        ref_o, ref_s, ref_p, _ = c.expect(q[s], kn[s], vn[s], b, n, nxt, GAMMA)
        check_close(widen(out[s], c.dtype), ref_o, RTOL[c.dtype], f"output {s}")
        left = int(after[6][s])
        assert after[7][s] == nxt + 1 and after[8][s] == 0
        assert left == (min(n + 1, int(lp.budget[s])) if lp.age_h[s] % INTERVAL == 0 else n + 1)
        for l in range(c.L):  # each position that is left has its own score
            of = dict(zip(ref_p[l].tolist(), ref_s[l].tolist()))
            at = after[5][l, b: b + left].tolist()
            assert len(set(at)) == left and nxt in at
            check_rel(after[4][l, b: b + left], np.array([of[x] for x in at]), SCORE_RTOL, f"score {s}")


@pytest.mark.parametrize("shape", [(BF16, 128, 8, 2, 3), (F32, 64, 6, 3, 2)])
def test_steps_match_the_oracle_and_a_request_joins(shape):
    lp, c = _loop(shape)
    dtype, d, Hq, Hkv, L = shape
    rng = np.random.default_rng(3)
    for step in range(STEPS):
        if step == 2:
            lp.retire(0)
        if step == 3:
            off = _spans(rng, 700)
            k, v = (store(rng.standard_normal((L, Hkv, 700, d)), dtype) for _ in "kv")
            assert lp.admit(0, to_dev(k), to_dev(v), to_dev(off), budget=170) == 175
            got = [from_dev(x[:, :, : 175]) for x in lp.planes]
            for x, y in zip(got, q4ref.span_means(widen(k, dtype), off) + q4ref.span_means(widen(v, dtype), off)):
                assert np.array_equal(x, y)
        before = _state(lp)
        q, kn, vn = c.rows(3)
        lp.step(to_dev(q), to_dev(kn), to_dev(vn))
        _check_step(lp, c, before, q, kn, vn, from_dev(lp.out))


@pytest.mark.parametrize("per_layer", [False, True])
@pytest.mark.parametrize("shape", [(BF16, 128, 8, 2, 3), (F32, 64, 6, 3, 2)])
def test_replayed_steps_are_the_eager_steps(shape, per_layer):
    t = torch()
    (eager, c), (graph, _) = _loop(shape), _loop(shape)
    dtype, d, Hq, Hkv, L = shape
    lead = (L, 3, 1) if per_layer else (3, L)
    bufs = [t.zeros(*lead, h, d, dtype=eager.out.dtype, device="cuda") for h in (Hq, Hkv, Hkv)]
    mix = t.zeros_like(bufs[0])

    def layer_query(l, q, outs):  # layer l's query depends on layer l - 1's output
        return q[0] if l == 0 else t.add(q[l], outs[l - 1], out=mix[l])

    graph.capture(*bufs, layer_query if per_layer else None)
    for a, b in zip(_state(eager)[:-1], _state(graph)):
        assert np.array_equal(a, b), "capture changed the state"
    for step in range(STEPS):
        rows = c.rows(3)
        if per_layer:
            rows = [np.ascontiguousarray(np.transpose(x, (1, 0, 2, 3))[:, :, None]) for x in rows]
        rows = [to_dev(x) for x in rows]
        eager.step(*rows, layer_query if per_layer else None)
        for b, x in zip(bufs, rows):
            b.copy_(x)
        graph.replay()
        _ = (rows[0].float() * 2).sum().item()  # eager work between replays
        for a, b in zip(_state(eager), _state(graph)):
            assert np.array_equal(a, b), f"step {step}"
        for a, b in zip(eager.out_layers + [eager.out], graph.out_layers + [graph.out]):
            assert t.equal(a, b)
    assert (from_dev(graph.length) <= np.array(BUDGETS) + INTERVAL).all()


def test_bits_are_4_or_the_rows_own():
    from paper_2608_08569_amd.loop import DecodeLoop
    with pytest.raises(ValueError, match="bits"):
        DecodeLoop(1, 1, 1, 64, [4], [2], 0.9, bits=8)
