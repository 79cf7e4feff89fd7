"""The 4-bit cache's work whose time is measured: calls as a serving program makes them.

A 4-bit cache holds K and V rows as e2m1 codes (two to a byte, the even channel
low) with one power-of-two scale per 32 channels, stored as a byte: scale byte b
stands for 2^(b - 127).  The kinds of pass:

  step     voxzip_decode_evict_q4: one generation step of one sequence at its
           budget (append, attention, decayed score, one row evicted)
  decode   voxzip_decode_attend_score_q4: the same without eviction
  ragged   voxzip_decode_attend_score_q4_ragged: one decode step of a batch of
           sequences of mixed lengths in one packed cache
  fuse     voxzip_fuse_spans_q4 over the prefill's K and V, and the rows read
           back by voxzip_unpack_q4
  prefill  fusion of a prefill, its attention mass as scores, the eviction down
           to the budget (voxzip_evict_compact_q4), and the rows read back
  admit    the same for a batch of requests, by the ragged twins

With `own` false, run() computes the same in plain torch operations.  The
decode kinds return the cache as it is held (codes and scales, which have to be
equal), the others the values that it stands for, which bfloat16 holds exactly.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

GAMMA = 0.95
N_SINK = 4
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the smallest call: a toy decoder's one float32 layer, 128 slots
        {"name": "step_f32_tiny", "kind": "step", "dtype": "f32", "L": 1, "Hq": 4, "Hkv": 1, "d": 64, "budget": 128},
        # one layer of a 4x-compressed 4k-token cache (a model that calls layer by layer)
        {"name": "step_layer", "kind": "step", "dtype": "bf16", "L": 1, "Hq": 32, "Hkv": 4, "d": 128, "budget": 1024},
        # the 32k-context cache at its 8192-slot budget, every layer in one call
        {"name": "step_long32k", "kind": "step", "dtype": "bf16", "L": 48, "Hq": 32, "Hkv": 4, "d": 128,
         "budget": 8192},
        # a model evaluated in full precision over a 4-bit cache
        {"name": "step_f32", "kind": "step", "dtype": "f32", "L": 16, "Hq": 16, "Hkv": 4, "d": 128, "budget": 2048},
        # a small decoder with head size 64 and groups of seven heads
        {"name": "decode_d64", "kind": "decode", "dtype": "bf16", "L": 24, "Hq": 14, "Hkv": 2, "d": 64, "T": 4001},
        # the fused 64k-token cache before its first eviction
        {"name": "decode_13k", "kind": "decode", "dtype": "bf16", "L": 48, "Hq": 32, "Hkv": 4, "d": 128, "T": 13181},
        # a batch of eight requests, every layer in one call
        {"name": "ragged_8", "kind": "ragged", "dtype": "bf16", "L": 48, "Hq": 32, "Hkv": 4, "d": 128, "n": 8,
         "lo": 1000, "hi": 8000},
        # one layer of a batch of sixteen requests (the model calls layer by layer)
        {"name": "ragged_16_layer", "kind": "ragged", "dtype": "bf16", "L": 1, "Hq": 32, "Hkv": 4, "d": 128, "n": 16,
         "lo": 1200, "hi": 8100},
        # the start of a 32k-token request
        {"name": "fuse_long32k", "kind": "fuse", "dtype": "bf16", "L": 48, "Hq": 32, "Hkv": 4, "d": 128,
         "T": 32768, "mean": 4.02, "anchor": False},
        # a short float32 prefill of a small decoder, with text anchors
        {"name": "fuse_f32_anchor", "kind": "fuse", "dtype": "f32", "L": 2, "Hq": 14, "Hkv": 2, "d": 64,
         "T": 4999, "mean": 3.1, "anchor": True},
        # one layer's 64k-token prefill, fused and cut to 5 % as the prefill passes that layer
        {"name": "prefill_64k", "kind": "prefill", "dtype": "bf16", "L": 1, "Hq": 32, "Hkv": 4, "d": 128,
         "T": 65536, "mean": 4.97, "budget": 3277},
        # four requests admitted together, each cut to a quarter of its spans
        {"name": "admit_4", "kind": "admit", "dtype": "bf16", "L": 12, "Hq": 32, "Hkv": 4, "d": 128, "n": 4,
         "lo": 2000, "hi": 9000, "mean": 4.02, "share": 0.25},
    ]


# ---- drawn cases ----

HEADS = [(4, 1), (8, 2), (14, 2), (16, 1), (16, 2), (16, 4), (32, 4), (32, 8), (64, 4), (64, 8)]
MOST_BYTES = 2e9


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "decode", "decode", "ragged", "ragged", "fuse", "prefill", "admit"])
    Hq, Hkv = rng.choice(HEADS)
    c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"]), "L": _logint(rng, 1, 48), "Hq": Hq, "Hkv": Hkv,
         "d": rng.choice([64, 128, 128])}
    if kind == "step":
        c["budget"] = _logint(rng, 96, 8192)
    elif kind == "decode":
        c["T"] = _logint(rng, 1, 32768)
    elif kind == "ragged":
        c["n"] = rng.randint(2, 24)
        c["lo"] = _logint(rng, 1, 3000)
        c["hi"] = c["lo"] + _logint(rng, 10, 8000)
    elif kind == "admit":
        c.update(L=rng.randint(1, 12), n=rng.randint(1, 8), lo=_logint(rng, 200, 5000),
                 mean=round(rng.uniform(1.5, 8.0), 2), share=round(rng.uniform(0.1, 0.9), 2))
        c["hi"] = c["lo"] + _logint(rng, 10, 8000)
    else:
        c["T"] = _logint(rng, 500, 65536)
        c["mean"] = round(rng.uniform(1.5, 8.0), 2)
        if kind == "prefill":
            c["L"] = rng.randint(1, 8)
            c["budget"] = max(32, int(_spans(c) * rng.uniform(0.1, 0.9)))
        else:
            c["anchor"] = rng.random() < 0.3
    while c["L"] > 1 and (work(c)["bytes"] > MOST_BYTES or _plain_bytes(c) > 2.5e9):
        c["L"] = (c["L"] + 1) // 2
    return c


# ---- sizes ----

def _spans(case):
    return max(1, int(round(case["T"] / case["mean"])))


def _lens(case):
    """Lengths of a batch's sequences, spread over [lo, hi] by their logarithm,
    the longest neither first nor last."""
    n = case["n"]
    x = np.exp(np.linspace(math.log(case["lo"]), math.log(case["hi"]), n)).astype(np.int64)
    x += np.arange(n) % 7  # not all of one parity
    return x[np.argsort((np.arange(n) * 7919 + 3) % (n + 1), kind="stable")]


def _batch(case):
    """Tokens, spans and budgets of the requests of an admitted batch."""
    T = _lens(case)
    n = np.maximum(1, np.round(T / case["mean"])).astype(np.int64)
    return T, n, np.maximum(8, (n * case["share"]).astype(np.int64))


def _keys(case):
    """Keys per layer that one pass attends over (the appended ones included)."""
    if case["kind"] == "step":
        return case["budget"] + 1
    return case["T"] if case["kind"] == "decode" else int((_lens(case) + 1).sum())


def _plain_bytes(case):
    """float32 bytes of the K rows that a plain pass holds at once (a batch padded to its longest)."""
    if case["kind"] == "ragged":
        keys = case["n"] * (int(_lens(case).max()) + 1)
    elif case["kind"] in ("step", "decode"):
        keys = _keys(case)
    else:
        keys = int(_lens(case).sum()) if case["kind"] == "admit" else case["T"]
    return 4 * case["L"] * case["Hkv"] * case["d"] * keys


def work(case):
    s = 2 if case["dtype"] == "bf16" else 4
    L, Hq, Hkv, d, kind = case["L"], case["Hq"], case["Hkv"], case["d"], case["kind"]
    full = 2 * Hkv * d * s            # K and V of one token in one layer, as the model gives them
    held = 2 * Hkv * (d // 2 + d // 32)  # the same in 4 bits with its scales
    if kind in ("fuse", "prefill", "admit"):
        if kind == "admit":
            T, n, budget = _batch(case)
            kept, T, n = float((budget * np.maximum(0, n - budget) / n).sum()), int(T.sum()), int(n.sum())
        else:
            T, n = case["T"], _spans(case)
            kept = case["budget"] * max(0, n - case["budget"]) / n if kind == "prefill" else 0.0
        # rows in, 4-bit rows with score and position out, then their values
        b = L * (T * full + n * (held + 8) + n * 2 * Hkv * d * 2)
        if case.get("anchor"):
            b += L * n * full
        if kind != "fuse":  # scores written and read with the positions, moved rows read and written
            b += L * (12 * n + 2 * kept * (held + 8))
        return {"bytes": b, "flops": 2 * L * T * Hkv * d}
    n, T = case.get("n", 1), _keys(case)
    b = L * (T * (held + 8) + n * (full + 2 * Hq * d * s))
    if kind == "step":  # positions read, one row moved
        b += L * (4 * T + 2 * (held + 8))
    return {"bytes": b, "flops": 4 * L * T * Hq * d}


# ---- inputs ----

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, *shape, dtype):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _kv(g, L, Hkv, T, d, dtype):
    """Keys or values: normal, with a scale per channel between 1/2 and 4."""
    x = _normal(g, L, Hkv, T, d, dtype=dtype)
    u = torch.rand(L, Hkv, 1, d, generator=g, device="cuda")
    return x.mul_(torch.exp(math.log(0.5) + u * math.log(8.0)).to(dtype))


def _scores(g, *shape):
    """Decayed attention sums: a heavy-tailed mass of about a few hundredths per key."""
    return torch.exp(2.0 * torch.randn(*shape, generator=g, device="cuda")).mul_(0.01)


def _positions(g, L, n, next_pos, recent):
    """Resident positions of a cache after evictions: the sinks, the recent
    window and a random choice of the others, in mixed slot order."""
    row = lambda m: torch.rand(L, m, generator=g, device="cuda").argsort(dim=1)
    first = torch.arange(N_SINK, device="cuda").expand(L, -1)
    last = torch.arange(next_pos - recent, next_pos, device="cuda").expand(L, -1)
    mid = row(next_pos - recent - N_SINK)[:, : n - N_SINK - recent] + N_SINK
    p = torch.cat([first, mid, last], 1)
    return p.gather(1, row(n)).int()


def _offsets(rng, T, n):
    """n contiguous spans over T tokens, cut at random: lengths about geometric."""
    cuts = rng.choice(T - 1, size=n - 1, replace=False) + 1
    return np.concatenate([[0], np.sort(cuts), [T]]).astype(np.int32)


def _i32(a):
    return torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()


def _i64(a):
    return torch.from_numpy(np.asarray(a, dtype=np.int64)).cuda()


def _zeros(dtype, *shape):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def _held(st, name, x):
    st[name + "_codes"], st[name + "_scales"] = _quantise(x)


def prepare(case, seed):
    g, dt = _gen(seed), DTYPE[case["dtype"]]
    kind, L, Hq, Hkv, d = case["kind"], case["L"], case["Hq"], case["Hkv"], case["d"]
    st = {"case": case}
    if kind in ("step", "decode"):
        n = case["budget"] if kind == "step" else case["T"] - 1
        cap = n + 2
        _held(st, "k", _kv(g, L, Hkv, cap, d, torch.float32))
        _held(st, "v", _kv(g, L, Hkv, cap, d, torch.float32))
        st.update(n=n, q=_normal(g, L, Hq, d, dtype=dt), kn=_kv(g, L, Hkv, 1, d, dt)[:, :, 0].contiguous(),
                  vn=_kv(g, L, Hkv, 1, d, dt)[:, :, 0].contiguous(), s=_scores(g, L, cap),
                  p=_zeros(torch.int32, L, cap), out=_zeros(dt, L, Hq, d))
        st["next"] = 2 * n if kind == "step" else n
        st["p"][:, :n] = (_positions(g, L, n, 2 * n, n // 5) if kind == "step"
                          else torch.arange(n, dtype=torch.int32, device="cuda"))
    elif kind == "ragged":
        lens = _lens(case)
        n, caps = case["n"], lens + 17
        total = int(caps.sum())
        base = np.concatenate([[0], np.cumsum(caps)[:-1]])
        _held(st, "k", _kv(g, L, Hkv, total, d, torch.float32))
        _held(st, "v", _kv(g, L, Hkv, total, d, torch.float32))
        st.update(q=_normal(g, n, L, Hq, d, dtype=dt), kn=_normal(g, n, L, Hkv, d, dtype=dt),
                  vn=_normal(g, n, L, Hkv, d, dtype=dt), s=_scores(g, L, total), p=_zeros(torch.int32, L, total),
                  out=_zeros(dt, n, L, Hq, d), base=_i64(base), cap=_i32(caps), len=_i32(lens), next=_i32(lens),
                  longest=int(lens.max()) + 1)
        for b, m in zip(base, lens):
            st["p"][:, int(b): int(b + m)] = torch.arange(int(m), dtype=torch.int32, device="cuda")
    elif kind == "admit":
        T, n, budget = _batch(case)
        rng = np.random.default_rng(seed)
        first = lambda x: np.concatenate([[0], np.cumsum(x)[:-1]])
        caps, total_in, S = n + 17, int(T.sum()), len(T)
        total = int(caps.sum())
        st.update(ki=_kv(g, L, Hkv, total_in, d, dt), vi=_kv(g, L, Hkv, total_in, d, dt), in_base=_i64(first(T)),
                  T_in=_i32(T), off=_i32(np.concatenate([_offsets(rng, t, m) for t, m in zip(T, n)])),
                  off_base=_i64(first(n + 1)), n_spans=_i32(n), max_spans=int(n.max()), base=_i64(first(caps)),
                  cap=_i32(caps), budget=_i32(budget), new_len=_zeros(torch.int32, S))
        slots = total
    else:
        T, n = case["T"], _spans(case)
        st.update(ki=_kv(g, L, Hkv, T, d, dt), vi=_kv(g, L, Hkv, T, d, dt), ak=None, av=None,
                  off=_i32(_offsets(np.random.default_rng(seed), T, n)))
        if case.get("anchor"):  # background spans carry no text: their anchors are zero rows
            text = (torch.rand(1, 1, n, 1, generator=g, device="cuda") < 0.7).to(dt)
            st.update(ak=_kv(g, L, Hkv, n, d, dt).mul_(text), av=_kv(g, L, Hkv, n, d, dt).mul_(text))
        slots = n + 2
    if kind in ("fuse", "prefill", "admit"):
        for x in "kv":
            st[x + "_codes"] = _zeros(torch.uint8, L, Hkv, slots, d // 2)
            st[x + "_scales"] = _zeros(torch.uint8, L, Hkv, slots, d // 32)
            st[x] = _zeros(torch.bfloat16, L, Hkv, slots, d)
        st.update(s=_zeros(torch.float32, L, slots), p=_zeros(torch.int32, L, slots))
        if kind != "fuse":
            st["mass"] = _scores(g, L, slots)
    return st


# ---- the plain form ----

def _quantise(x):
    """Rows [..., d] as codes [..., d / 2] and scale bytes [..., d / 32]: per 32
    channels the smallest power of two 2^e with max |x| <= 7 * 2^e (e within
    -125 .. 125), and x / 2^e to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (6 at
    most), ties to the even code."""
    b = x.unflatten(-1, (-1, 32))
    a = b.abs()
    top = a.amax(-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e with 1/2 <= m < 1
    e = torch.where(top > 0, e - 3 + (m > 0.875), -125).clamp(-125, 125)
    a = torch.ldexp(a, -e)
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte()
            + (a >= 3.5).byte() + (a > 5).byte() + 8 * (b < 0).byte()).flatten(-2)
    return code[..., ::2] + 16 * code[..., 1::2], (e + 127).squeeze(-1).byte()


def _values(codes, scales):
    """The float32 values that codes and scales stand for."""
    mag = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    one = torch.tensor(mag + [-m for m in mag], device=codes.device)
    pair = torch.stack([one.repeat(16), one.repeat_interleave(16)], 1)  # of each byte: low code, high code
    x = pair.index_select(0, codes.reshape(-1).int()).view(*scales.shape, 32)
    return (x * (scales.int() << 23).view(torch.float32).unsqueeze(-1)).flatten(-2)


def _attention(q, K, V, scale, mask=None):
    """q [..., G, d] over keys [..., T, d]: outputs and each key's sum over the heads of the probabilities."""
    z = torch.matmul(q, K.transpose(-1, -2)) * scale
    if mask is not None:
        z = z.masked_fill(~mask, -math.inf)
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    return torch.matmul(p, V), p.sum(-2)


def _plain_decode(st):
    n, out = st["n"], st["out"]
    L, Hq, d = out.shape
    Hkv = st["kn"].shape[1]
    for_slot = {"k": st["kn"], "v": st["vn"]}
    kc, ks = _quantise(for_slot["k"].float())
    vc, vs = _quantise(for_slot["v"].float())
    st["k_codes"][:, :, n], st["k_scales"][:, :, n] = kc, ks
    st["v_codes"][:, :, n], st["v_scales"][:, :, n] = vc, vs
    st["p"][:, n] = st["next"]
    K = _values(st["k_codes"][:, :, : n + 1], st["k_scales"][:, :, : n + 1])
    V = _values(st["v_codes"][:, :, : n + 1], st["v_scales"][:, :, : n + 1])
    o, mass = _attention(st["q"].float().view(L, Hkv, Hq // Hkv, d), K, V, 1 / math.sqrt(d))
    out.copy_(o.view(L, Hq, d))
    st["s"][:, n] = 0
    st["s"][:, : n + 1] = GAMMA * st["s"][:, : n + 1] + mass.sum(1)


def _order(score, pos, middle):
    """Slots of each row, the first to go first: the smallest score, of equal ones the larger position; sinks and
    recent ones last."""
    by_pos = pos.argsort(dim=-1, descending=True, stable=True)
    key = torch.where(middle, score, math.inf).gather(-1, by_pos)
    return by_pos.gather(-1, key.argsort(dim=-1, stable=True))


def _plain_evict(st, at, length, budget, next_pos):
    """Keeps `budget` of the first `length` of each sequence's slots at[s] (int64 [S, W]; length, budget and next_pos
    [S, 1]): the kept slots past the budget fill the freed ones below it, both in slot order."""
    W = at.shape[1]
    j = torch.arange(W, device=at.device)
    held = j < length
    pos, score = st["p"][:, at].long(), st["s"][:, at]
    middle = (pos >= N_SINK) & (pos < next_pos - budget // 5) & held
    order = _order(score, pos, middle)
    gone = torch.zeros_like(middle).scatter_(-1, order, (j < length - budget).expand_as(order)) & middle
    mover = (j >= budget) & held & ~gone
    hole = gone & (j < budget)
    movers = torch.where(mover, j, W).sort(-1).values  # in slot order
    fill = movers.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0))
    source = torch.where(hole & (fill < W), fill, j)  # [L, S, W]
    ok = held & (j < budget)
    to, of = at[ok], at.expand_as(source).gather(-1, source)[:, ok]
    layer = torch.arange(of.shape[0], device=at.device)[:, None]
    st["s"][:, to], st["p"][:, to] = st["s"][layer, of], st["p"][layer, of]
    head = torch.arange(st["k_codes"].shape[1], device=at.device)[:, None]
    here = (layer[:, :, None], head, of[:, None, :])
    st["k_codes"][:, :, to], st["k_scales"][:, :, to] = st["k_codes"][here], st["k_scales"][here]
    st["v_codes"][:, :, to], st["v_scales"][:, :, to] = st["v_codes"][here], st["v_scales"][here]


def _one(x):
    return torch.tensor([[x]], device="cuda")


def _plain_ragged(st):
    out, base, length = st["out"], st["base"], st["len"].long()
    S, L, Hq, d = out.shape
    Hkv = st["kn"].shape[2]
    new = base + length
    kc, ks = _quantise(st["kn"].float().permute(1, 2, 0, 3))
    vc, vs = _quantise(st["vn"].float().permute(1, 2, 0, 3))
    st["k_codes"][:, :, new], st["k_scales"][:, :, new] = kc, ks
    st["v_codes"][:, :, new], st["v_scales"][:, :, new] = vc, vs
    st["p"][:, new], st["s"][:, new] = st["next"], 0.0
    j = torch.arange(st["longest"], device=base.device)
    mask = j <= length[:, None]
    at = torch.where(mask, base[:, None] + j, base[:, None])
    K = _values(st["k_codes"][:, :, at], st["k_scales"][:, :, at])
    V = _values(st["v_codes"][:, :, at], st["v_scales"][:, :, at])
    q = st["q"].float().view(S, L, Hkv, Hq // Hkv, d).permute(1, 2, 0, 3, 4)
    o, mass = _attention(q, K, V, 1 / math.sqrt(d), mask[:, None, :])
    out.copy_(o.permute(2, 0, 1, 3, 4).reshape(S, L, Hq, d))
    st["s"][:, at[mask]] = GAMMA * st["s"][:, at[mask]] + mass.sum(1)[:, mask]


def _plain_means(x, anchor, first, span_of_row, count):
    """(sum of the span's rows + count * anchor) / count, in 64 bits: the codes of values at a border turn on it."""
    L, H, _, d = x.shape
    y = torch.zeros(L, H, first.shape[0], d, dtype=torch.float64, device=x.device)
    y.index_add_(2, span_of_row, x.double())
    if anchor is not None:
        y += count * anchor.double()
    return y / count


def _plain_fuse(st, first, rows, slot, pos):
    """Spans starting at rows `first` (ascending) of `rows` rows, to slots `slot` at positions `pos`."""
    mark = torch.zeros(rows, dtype=torch.int64, device=first.device)
    mark[first] = 1
    end = torch.cat([first[1:], torch.full_like(first[:1], rows)])
    where = (first, mark.cumsum(0) - 1, (end - first).double()[:, None])
    kc, ks = _quantise(_plain_means(st["ki"], st.get("ak"), *where))
    vc, vs = _quantise(_plain_means(st["vi"], st.get("av"), *where))
    st["k_codes"][:, :, slot], st["k_scales"][:, :, slot] = kc, ks
    st["v_codes"][:, :, slot], st["v_scales"][:, :, slot] = vc, vs
    st["s"][:, slot], st["p"][:, slot] = 0.0, pos.int()


def _plain(st):
    kind, case = st["case"]["kind"], st["case"]
    if kind in ("step", "decode"):
        _plain_decode(st)
        if kind == "step":
            B = case["budget"]
            _plain_evict(st, torch.arange(B + 1, device="cuda")[None], _one(B + 1), _one(B), _one(st["next"] + 1))
        st["next"] += 1
    elif kind == "ragged":
        _plain_ragged(st)
        st["next"].add_(1)
    elif kind == "admit":
        n, base = st["n_spans"].long(), st["base"]
        S, N = n.shape[0], st["off"].shape[0]
        seq = torch.repeat_interleave(torch.arange(S, device="cuda"), n + 1, output_size=N)
        j = torch.arange(N, device="cuda") - st["off_base"][seq]
        start = j < n[seq]  # the last offset of a sequence starts no span
        _plain_fuse(st, (st["off"] + st["in_base"][seq])[start], st["ki"].shape[2], (base[seq] + j)[start], j[start])
        st["s"].copy_(st["mass"])
        at = base[:, None] + torch.arange(st["max_spans"], device="cuda")
        held = at < (base + n)[:, None]
        _plain_evict(st, torch.where(held, at, base[:, None]), n[:, None], st["budget"].long()[:, None], n[:, None])
        st["new_len"].copy_(torch.minimum(st["n_spans"], st["budget"]))
    else:
        n = st["off"].shape[0] - 1
        j = torch.arange(n, device="cuda")
        _plain_fuse(st, st["off"][:-1].long(), case["T"], j, j)
        if kind == "prefill":
            st["s"].copy_(st["mass"])
            _plain_evict(st, j[None], _one(n), _one(case["budget"]), _one(n))
    if kind in ("fuse", "prefill", "admit"):
        st["k"].copy_(_values(st["k_codes"], st["k_scales"]))
        st["v"].copy_(_values(st["v_codes"], st["v_scales"]))


# ---- one pass ----

def _workspace(vz, st, op, ragged=False):
    """The call's scratch memory, made once and kept, as a program keeps it."""
    if "ws" not in st:
        L, Hkv, slots, half = st["k_codes"].shape
        make, more = (vz.workspace_ragged, (st["base"].shape[0],)) if ragged else (vz.workspace, ())
        st["ws"] = make(op, L, st["case"]["Hq"], Hkv, 2 * half, slots, *more)
    return st["ws"]


def _calls(st):
    import paper_2608_08569_amd as vz
    case = st["case"]
    kind = case["kind"]
    if kind == "step":
        vz.voxzip_decode_evict_q4(st["q"], st["kn"], st["vn"], st["k_codes"], st["k_scales"], st["v_codes"],
                                  st["v_scales"], st["s"], st["p"], st["out"], st["n"], st["next"], GAMMA,
                                  case["budget"], n_sink=N_SINK, workspace=_workspace(vz, st, vz.VZ_OP_DECODE_EVICT_Q4))
        st["next"] += 1
    elif kind == "decode":
        vz.voxzip_decode_attend_score_q4(st["q"], st["kn"], st["vn"], st["k_codes"], st["k_scales"], st["v_codes"],
                                         st["v_scales"], st["s"], st["p"], st["out"], st["n"], st["next"], GAMMA,
                                         workspace=_workspace(vz, st, vz.VZ_OP_DECODE_Q4))
        st["next"] += 1
    elif kind == "ragged":
        vz.voxzip_decode_attend_score_q4_ragged(st["q"], st["kn"], st["vn"], st["k_codes"], st["k_scales"],
                                                st["v_codes"], st["v_scales"], st["s"], st["p"], st["out"],
                                                st["base"], st["cap"], st["len"], st["next"], GAMMA,
                                                workspace=_workspace(vz, st, vz.VZ_OP_DECODE_Q4, ragged=True))
        st["next"].add_(1)
    elif kind == "admit":
        vz.voxzip_fuse_spans_q4_ragged(st["ki"], st["vi"], st["in_base"], st["T_in"], st["off"], st["off_base"],
                                       st["n_spans"], st["max_spans"], st["k_codes"], st["k_scales"], st["v_codes"],
                                       st["v_scales"], st["s"], st["p"], st["base"], st["cap"])
        st["s"].copy_(st["mass"])
        vz.voxzip_evict_compact_q4_ragged(st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"], st["s"],
                                          st["p"], st["base"], st["cap"], st["n_spans"], st["budget"],
                                          st["n_spans"], n_sink=N_SINK, new_len_out=st["new_len"],
                                          workspace=_workspace(vz, st, vz.VZ_OP_EVICT, ragged=True))
    else:
        vz.voxzip_fuse_spans_q4(st["ki"], st["vi"], st["off"], st["k_codes"], st["k_scales"], st["v_codes"],
                                st["v_scales"], st["s"], st["p"], anchor_k=st["ak"], anchor_v=st["av"])
        if kind == "prefill":
            n = st["off"].shape[0] - 1
            st["s"].copy_(st["mass"])
            vz.voxzip_evict_compact_q4(st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"], st["s"],
                                       st["p"], n, case["budget"], n, n_sink=N_SINK,
                                       workspace=_workspace(vz, st, vz.VZ_OP_EVICT))
    if kind in ("fuse", "prefill", "admit"):
        vz.voxzip_unpack_q4(st["k_codes"], st["k_scales"], st["k"])
        vz.voxzip_unpack_q4(st["v_codes"], st["v_scales"], st["v"])


def run(st):
    if own:
        _calls(st)
    else:
        _plain(st)
    got = {"score": st["s"], "pos": st["p"]}
    if st["case"]["kind"] in ("fuse", "prefill", "admit"):
        got.update(k=st["k"], v=st["v"])
        if st["case"]["kind"] == "admit":
            got["new_len"] = st["new_len"]
    else:
        got.update({x: st[x] for x in ("out", "k_codes", "k_scales", "v_codes", "v_scales")})
    return got


# ---- the same in 64 bits, from the definition ----

def _nearest(x):
    """x [..., d] rounded as a 4-bit cache holds it, the scale by comparison and the value by its binade's step."""
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    top = b.abs().max(-1, keepdim=True).values
    e = (torch.log2(top) - 5).floor().clamp(-125, 125)  # below the scale that is sought
    for _ in range(4):
        e = e + ((top > 7 * torch.exp2(e)) & (e < 125))
    a = b.abs() / torch.exp2(e)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    r = torch.clamp(torch.round(a / step) * step, max=6.0)  # round(): halves to even
    return (torch.sign(b) * r * torch.exp2(e)).reshape(x.shape)


def _read(codes, scales):
    """What codes and scales stand for: sign, exponent and mantissa bits of each code."""
    c = torch.stack([codes % 16, codes // 16], -1).flatten(-2).double()
    sign, exp, man = 1 - 2 * (c >= 8).double(), (c % 8) // 2, c % 2
    x = sign * torch.where(exp > 0, torch.exp2(exp - 1) * (1 + man / 2), man / 2)
    return x * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def _attend(q, kn, vn, kc, ks, vc, vs, s):
    """One layer of one sequence: the n keys held and the new one; output and decayed scores of the n + 1 slots."""
    Hq, d = q.shape
    Hkv = kn.shape[0]
    K = torch.cat([_read(kc, ks), _nearest(kn)[:, None]], 1)
    V = torch.cat([_read(vc, vs), _nearest(vn)[:, None]], 1)
    a = torch.softmax(torch.bmm(q.double().view(Hkv, Hq // Hkv, d), K.transpose(1, 2).contiguous()) / math.sqrt(d), -1)
    old = torch.cat([s.double(), torch.zeros(1, dtype=torch.float64, device=s.device)])
    return torch.bmm(a, V).view(Hq, d), GAMMA * old + a.sum((0, 1))


def _kept_moves(score, pos, n, budget, next_pos):
    """Slots to fill and the slots that fill them, in slot order."""
    p, s = pos[:n].cpu().numpy().astype(np.int64), score[:n].cpu().numpy()
    order = np.lexsort((-p, s))  # smallest score first, then the larger position
    mid = (p >= N_SINK) & (p < next_pos - budget // 5)
    gone = np.zeros(n, dtype=bool)
    gone[order[mid[order]][: max(0, n - budget)]] = True
    holes, movers = np.flatnonzero(gone[:budget]), np.flatnonzero(~gone[budget:]) + budget
    m = min(len(holes), len(movers))
    return _i64(holes[:m]), _i64(movers[:m])


def _fused(x, anchor, off):
    """One layer's spans: the mean of each one's rows and its anchor, as a 4-bit cache holds it."""
    first, size = off[:-1].long(), (off[1:] - off[:-1]).long()
    y = torch.zeros(x.shape[0], first.shape[0], x.shape[-1], dtype=torch.float64, device=x.device)
    for k in range(int(size.max())):
        on = size > k
        y[:, on] += x[:, first[on] + k].double()
    m = size.double()[:, None]
    return _nearest((y + (0 if anchor is None else anchor.double() * m)) / m)


def exact(case, seed):
    kind, L = case["kind"], case["L"]
    st = prepare(case, seed)
    held = [st["k_codes"], st["k_scales"], st["v_codes"], st["v_scales"]]
    none = {"pos": None, "k_codes": None, "k_scales": None, "v_codes": None, "v_scales": None}
    if kind == "ragged":
        out, s = st["out"].double(), st["s"].double()
        for i, (b, n) in enumerate(zip(st["base"].tolist(), st["len"].tolist())):
            for l in range(L):
                out[i, l], s[l, b: b + n + 1] = _attend(st["q"][i, l], st["kn"][i, l], st["vn"][i, l],
                                                       *(x[l, :, b: b + n] for x in held), st["s"][l, b: b + n])
        return {"out": out, "score": s, **none}
    if kind in ("step", "decode"):
        n = st["n"]
        out, s = st["out"].double(), st["s"].double()
        for l in range(L):
            out[l], s[l, : n + 1] = _attend(st["q"][l], st["kn"][l], st["vn"][l], *(x[l, :, :n] for x in held),
                                            st["s"][l, :n])
            if kind == "step":
                pos = torch.cat([st["p"][l, :n], torch.tensor([st["next"]], dtype=torch.int32, device="cuda")])
                holes, movers = _kept_moves(s[l], pos, n + 1, case["budget"], st["next"] + 1)
                s[l, holes] = s[l, movers]
        return {"out": out, "score": s, **none}
    k, v = (torch.zeros_like(st[x], dtype=torch.float64) for x in "kv")
    if kind == "admit":
        rows = list(zip(*(st[x].tolist() for x in ("in_base", "T_in", "off_base", "n_spans", "base", "budget"))))
    else:
        rows = [(0, case["T"], 0, _spans(case), 0, case.get("budget", 1 << 30))]
    for ib, T, ob, n, b, budget in rows:
        off = st["off"][ob: ob + n + 1]
        for l in range(L):
            for x, y, a in ((st["ki"], k, st.get("ak")), (st["vi"], v, st.get("av"))):
                y[l, :, b: b + n] = _fused(x[l, :, ib: ib + T], None if a is None else a[l], off)
            if kind != "fuse":
                pos = torch.arange(n, dtype=torch.int32, device="cuda")
                holes, movers = _kept_moves(st["mass"][l, b: b + n], pos, n, budget, n)
                for y in (k, v):
                    y[l][:, b + holes] = y[l][:, b + movers]
    return {"k": k, "v": v, "score": None, "pos": None, "new_len": None}
