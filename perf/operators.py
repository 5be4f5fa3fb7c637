"""Timed cases of the operators that shrink a cache: 8-bit codes, and eviction by
accumulated attention weight.

Every case is one call of one attention layer of a serving program:

  pack    quantize_kv of rows that a program has in 16 or 32 bits: a pool's
          caches, a route-compacted store, or a prompt's projections
  append  quantize_kv of the newest tokens of running conversations
  attend  attend_quantized: prefill (several queries per request) or decode
          (one) over routed resources and context, all in 8 bits
  weigh   attend_weights: what every cached row has been attended to
  evict   select_kept: the rows of every segment that stay

Where `own` is false the cases run in plain torch operations of 32 bits (64 for
the sums that a selection compares); where it is true, through the package.
"""
import math
import zlib

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 64      # tokens that share a scale
F8 = torch.float8_e4m3fn

ATTEND = dict(dtype="bf16", hq=32, hkv=8, d=128, n_req=8, per_req=8, pool=64, len_lo=300, len_hi=1200,
              keep=1.0, routes=1.0, q_lo=2048, q_hi=2048, past_lo=0, past_hi=0, slack=0, store=False)
PRUNED = dict(keep=0.3, routes=0.25)
EVICT = dict(kind="evict", n_seg=64, len_lo=300, len_hi=1200, planes=8, keep=0.3, first=0, last=1)


def listed():
    return [
        # the newest token of one conversation joins its 8-bit context: latency
        dict(ATTEND, name="append_one", kind="append", n_req=1, pool=0, per_req=0, q_lo=1, q_hi=1,
             past_lo=3000, past_hi=3000, slack=500),
        # one decode step's tokens of a full batch
        dict(ATTEND, name="append_batch", kind="append", n_req=64, pool=0, per_req=0, q_lo=1, q_hi=1,
             past_lo=60, past_hi=9000, slack=128),
        # a whole layer of a large route-compacted store is put into 8 bits
        dict(ATTEND, **PRUNED, name="pack_store", kind="pack", pool=2048, per_req=32, n_req=64, len_lo=200,
             len_hi=2000, store=True, source="cache"),
        # one new token of one conversation with eight tools: latency
        dict(ATTEND, **PRUNED, name="decode_one", kind="attend", n_req=1, pool=8, q_lo=1, q_hi=1,
             past_lo=3000, past_hi=3000, store=True, slack=200),
        # a moderate batch, contexts of very unequal length, shared tools, 16 / 8 heads
        dict(ATTEND, **PRUNED, name="decode_ragged", kind="attend", hq=16, n_req=12, per_req=12, pool=48,
             len_lo=100, q_lo=1, q_hi=1, past_lo=60, past_hi=9000, store=True),
        # full-rate batched decode: 64 conversations over 32 tools each
        dict(ATTEND, **PRUNED, name="decode_batch", kind="attend", n_req=64, per_req=32, pool=2048, len_lo=200,
             len_hi=2000, q_lo=1, q_hi=1, past_lo=4095, past_hi=4095),
        # a user's next message in a running conversation
        dict(ATTEND, **PRUNED, name="turn_one", kind="attend", n_req=1, pool=8, q_lo=75, q_hi=75, past_lo=2600,
             past_hi=2600),
        # first pass over long prompts, everything visible: the largest call
        dict(ATTEND, name="prefill_full", kind="attend"),
        # a decode step adds to what each cached row has been attended to
        dict(ATTEND, **PRUNED, name="weigh_decode", kind="weigh", n_req=64, per_req=32, pool=256, len_lo=200,
             len_hi=2000, q_lo=1, q_hi=1, past_lo=4095, past_hi=4095, prior=True),
        # a prompt scores the tools it was given, before they are pruned
        dict(ATTEND, name="weigh_prompt", kind="weigh", prior=False),
        # every tool of a pool keeps the best 30% of its tokens
        dict(EVICT, name="evict_pool", n_seg=2048, len_lo=200, len_hi=2000),
        # long conversations keep a quarter, the first and the newest tokens among it
        dict(EVICT, name="evict_context", n_seg=6, len_lo=12000, len_hi=100000, keep=0.25, first=4, last=64),
    ]


def _span(rng, lo, hi):
    """A whole number, uniform in its logarithm over lo .. hi."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "pack", "decode", "decode", "prefill", "prefill", "weigh", "weigh", "evict"))
    if kind == "evict":
        n = _span(rng, 1, 1500)
        lo = _span(rng, 1, 300)
        return dict(EVICT, n_seg=n, len_lo=lo, len_hi=lo + _span(rng, 1, min(60000, 1500000 // n)),
                    planes=rng.choice((1, 4, 8, 8)), keep=rng.choice((0.05, 0.3, 0.7)),
                    first=rng.choice((0, 4)), last=rng.choice((0, 1, 32)))
    hq, hkv, d = rng.choice(((32, 8, 128), (32, 8, 128), (16, 8, 128), (28, 4, 128), (64, 8, 128),
                             (8, 8, 128), (8, 2, 64), (12, 4, 64)))
    lo = _span(rng, 20, 400)
    case = dict(ATTEND, hq=hq, hkv=hkv, d=d, len_lo=lo, len_hi=lo + _span(rng, 1, 1500),
                **(PRUNED if rng.random() < 0.6 else {}))
    per = _span(rng, 1, 24)
    n = _span(rng, 1, 64)
    if kind == "append":
        return dict(case, kind=kind, n_req=n, pool=0, per_req=0, q_lo=1, q_hi=rng.choice((1, 1, 40)),
                    past_lo=0, past_hi=_span(rng, 64, 9000), slack=rng.choice((0, 200)),
                    dtype=rng.choice(("bf16", "bf16", "f32")))
    if kind == "pack":
        return dict(case, kind=kind, n_req=n, per_req=per, pool=max(per, _span(rng, 1, 150)), q_lo=1,
                    q_hi=_span(rng, 2, 2000), store=rng.random() < 0.5, source=rng.choice(("cache", "prompt")),
                    dtype=rng.choice(("bf16", "bf16", "f32")))
    if kind == "decode" or (kind == "weigh" and rng.random() < 0.5):
        case.update(n_req=n, per_req=per, pool=max(per, _span(rng, 1, 200)), q_lo=1, q_hi=1,
                    past_lo=_span(rng, 1, 2000), past_hi=_span(rng, 2000, 160000 // (n + 12)))
    else:
        n = _span(rng, 1, 10)
        q = min(_span(rng, 2, 2048), 16000 // n, 260000 // (hq * n) + 2)
        per = min(per, 12)
        case.update(n_req=n, per_req=per, pool=per + rng.randrange(40), q_lo=max(1, q // rng.choice((1, 4, 30))),
                    q_hi=q, past_lo=0, past_hi=_span(rng, 1, 4000))
    case["store"] = rng.random() < 0.5
    if kind == "weigh":
        return dict(case, kind=kind, prior=rng.random() < 0.5,
                    dtype=rng.choice(("bf16", "bf16", "f32")) if case["q_hi"] * case["n_req"] < 2000 else "bf16")
    return dict(case, kind="attend", slack=rng.choice((0, 0, 200)))


# ------------------------------------------------------------------ structure

def _prefix(a):
    return np.concatenate([[0], np.cumsum(np.asarray(a, np.int64))])


def _rng(case):
    return np.random.default_rng(zlib.crc32(repr(sorted(case.items())).encode()))


def _spread(rng, lo, hi, n):
    """Lengths over lo .. hi, over their logarithm where the range is wide."""
    if hi > 10 * lo:
        return np.round(np.exp(rng.uniform(math.log(lo), math.log(hi), n))).astype(np.int64)
    return rng.integers(lo, hi + 1, n)


def _evict_structure(case):
    rng = _rng(case)
    S = {"len": _spread(rng, case["len_lo"], case["len_hi"], case["n_seg"])}
    S["cu"] = _prefix(S["len"])
    S["k"] = np.maximum(1, np.floor(case["keep"] * S["len"] + 0.5).astype(np.int64))
    S["cu_kept"] = _prefix(S["k"])
    return S


def _structure(case):
    """Host-side lengths, request lists and routes of one layer.  Resource r
    has rows[r] cached rows; seg_cu are the offsets of the cache's segments:
    the resources, or in a store the routes (r, g) in that order."""
    rng = _rng(case)
    G, n, per = case["hkv"], case["n_req"], case["per_req"]
    S = {}
    length = rng.integers(case["len_lo"], case["len_hi"] + 1, case["pool"])
    S["rows"] = np.maximum(1, np.floor(case["keep"] * length + 0.5).astype(np.int64))
    S["cu_kept"] = _prefix(S["rows"])
    S["mask"] = (rng.random((case["pool"], G)) < case["routes"]).astype(np.uint8)
    if n * per == case["pool"]:
        S["lists"] = np.arange(case["pool"]).reshape(n, per)
    else:
        S["lists"] = np.stack([rng.permutation(case["pool"])[:per] for _ in range(n)]).reshape(n, per)
    S["seg_cu"] = _prefix((S["rows"][:, None] * S["mask"]).reshape(-1)) if case["store"] else S["cu_kept"]
    S["q"] = rng.integers(case["q_lo"], case["q_hi"] + 1, n)
    S["ctx"] = S["q"] + (_spread(rng, case["past_lo"], case["past_hi"], n) if case["past_lo"] > 0 else
                         rng.integers(case["past_lo"], case["past_hi"] + 1, n))
    S["cu_q"], S["cu_ctx"] = _prefix(S["q"]), _prefix(S["ctx"] + case["slack"])
    # route lists of (request, group), and the tokens they hold
    seen = S["mask"][S["lists"]] != 0                                   # [n][per][G]
    S["route_off"] = _prefix(seen.sum(1).reshape(-1))
    S["route_res"] = np.concatenate([S["lists"][b][seen[b, :, g]] for b in range(n) for g in range(G)] or [[]])
    S["vis"] = (S["rows"][S["lists"]][:, :, None] * seen).sum(1)         # [n][G]
    # users of every resource, in request order
    order = np.argsort(S["lists"].reshape(-1), kind="stable")
    S["user_req"] = order // max(per, 1)
    S["user_off"] = _prefix(np.bincount(S["lists"].reshape(-1), minlength=case["pool"]))
    return S


def _slots(cu, lens):
    """For every row of every segment in turn: its cache row, its scale's slot
    and its place in the segment."""
    at = np.concatenate([np.arange(n) for n in lens] or [[]]).astype(np.int64)
    seg = np.repeat(np.arange(len(lens)), lens)
    return cu[seg] + at, cu[seg] // BLOCK + seg + at // BLOCK, at


def _n_slots(rows, n_seg):
    return rows // BLOCK + n_seg


def _key_rows(case, S, b):
    """Rows (in a cache's planes laid end to end) and scale slots of request
    b's resource keys, [G][m], and which of them each group sees."""
    G, mine = case["hkv"], S["lists"][b]
    n = S["rows"][mine]
    at = np.concatenate([np.arange(x) for x in n] or [[]]).astype(np.int64)
    r = np.repeat(mine, n)
    g = np.arange(G)[:, None]
    seen = S["mask"][r].T != 0 if len(r) else np.zeros((G, 0), bool)
    n_seg, total = len(S["seg_cu"]) - 1, int(S["seg_cu"][-1])
    seg = r[None] * G + g if case["store"] else np.broadcast_to(r[None], (G, len(r)))
    row = S["seg_cu"][seg] + at
    slot = S["seg_cu"][seg] // BLOCK + seg + at // BLOCK
    if not case["store"]:
        row, slot = row + g * total, slot + g * _n_slots(total, n_seg)
    return np.where(seen, row, 0), np.where(seen, slot, 0), seen


# ------------------------------------------------------------------ prepare

def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(dtype))).to(DEV)


class _Normal:
    """Seeded N(0, 1) tensors on the GPU, one after another; keys have a few
    channels of larger spread, as a model's do."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def __call__(self, *shape, dtype=torch.float32):
        return torch.randn(*shape, generator=self.g, device=DEV, dtype=dtype)

    def keys(self, *shape, dtype=torch.float32):
        x = self(*shape, dtype=dtype)
        x[..., 1::shape[-1] // 4] *= 3
        return x


def _cache8(N, keys, planes, cu, lens, d):
    """A cache in 8 bits: codes [planes][rows][d] and exponents [planes][slots]."""
    rows, n_seg = int(cu[-1]), len(cu) - 1
    codes = torch.zeros(planes, rows, d, dtype=torch.uint8, device=DEV)
    exps = torch.zeros(planes, _n_slots(rows, n_seg), dtype=torch.uint8, device=DEV)
    at, slot, _ = _slots(cu, lens)
    at, slot = _dev(at, np.int64), _dev(slot, np.int64)
    for p in range(planes):
        x = N.keys(len(at), d) if keys else N(len(at), d)
        c, e = _quantize(x.to(torch.bfloat16)[None], slot, torch.ones(1, exps.shape[1], dtype=torch.int32, device=DEV))
        codes[p, at] = c[0].view(torch.uint8)
        exps[p] = e[0].to(torch.uint8)
    return codes.view(F8), exps


def prepare(case, seed):
    N = _Normal(seed)
    if case["kind"] == "evict":
        S = _evict_structure(case)
        w = N(case["planes"], int(S["cu"][-1])).exp_()
        # rows that nothing attended to, the same in every plane
        w *= torch.rand(1, w.shape[1], generator=N.g, device=DEV) > 0.1
        j = np.concatenate([np.arange(x) for x in S["len"]])
        n, k = np.repeat(S["len"], S["len"]), np.repeat(S["k"], S["len"])
        last = np.minimum(case["last"], k)
        forced = (j >= n - last) | (j < np.minimum(case["first"], k - last))
        return {"case": case, "w": w, "cu": _dev(S["cu"]), "cu_kept": _dev(S["cu_kept"]), "max_len": int(S["len"].max()),
                "seg": _dev(np.repeat(np.arange(len(S["len"])), S["len"]), np.int64), "forced": _dev(forced, np.bool_),
                "kept": torch.zeros(int(S["cu_kept"][-1]), dtype=torch.int32, device=DEV),
                "kept_w": torch.zeros(case["planes"], int(S["cu_kept"][-1]), device=DEV), "ws": {}}
    S = _structure(case)
    G, d, hq, n = case["hkv"], case["d"], case["hq"], case["n_req"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    st = {"case": case, "cu_q": _dev(S["cu_q"]), "cu_ctx": _dev(S["cu_ctx"]), "cu_kept": _dev(S["cu_kept"]),
          "len": _dev(S["ctx"]) if case["slack"] else None}
    if case["kind"] in ("pack", "append"):
        return _prepare_quantize(case, S, N, dt, st)
    st["route"] = tuple(_dev(S[x]) for x in ("route_off", "route_res", "vis"))
    st["res_off"] = _dev(S["seg_cu"]) if case["store"] else None
    st["q"] = N(int(S["cu_q"][-1]), hq, d, dtype=dt)
    st["max_q"], st["max_ctx"] = int(S["q"].max()), int(S["ctx"].max())
    st["max_kv"] = int((S["vis"].max(1) + S["ctx"]).max())
    # what the plain form needs to know of every request
    st["req"] = []
    for b in range(n):
        row, slot, seen = _key_rows(case, S, b)
        st["req"].append((int(S["cu_q"][b]), int(S["q"][b]), int(S["cu_ctx"][b]), int(S["ctx"][b]),
                          _dev(row, np.int64), _dev(slot, np.int64), _dev(seen, np.bool_)))
    planes = 1 if case["store"] else G
    seg_len = np.diff(S["seg_cu"])
    if case["kind"] == "attend":
        st["rk"], st["rk_exp"] = _cache8(N, True, planes, S["seg_cu"], seg_len, d)
        st["rv"], st["rv_exp"] = _cache8(N, False, planes, S["seg_cu"], seg_len, d)
        st["ck"], st["ck_exp"] = _cache8(N, True, G, S["cu_ctx"], S["ctx"], d)
        st["cv"], st["cv_exp"] = _cache8(N, False, G, S["cu_ctx"], S["ctx"], d)
        _, slot, _ = _slots(S["cu_ctx"], S["ctx"])
        st["ctx_slot"] = [_dev(x, np.int64) for x in np.split(slot, _prefix(S["ctx"])[1:-1])]
        if case["store"]:
            for x in ("rk", "rv", "rk_exp", "rv_exp"):
                st[x] = st[x][0]
        st["out"] = torch.zeros_like(st["q"])
        # at most 64 splits of every request's keys
        st["ws"] = torch.empty(n * hq * 64 * (d + 2), device=DEV) if st["max_q"] == 1 else None
        return st
    st["rk"] = N.keys(*(() if case["store"] else (G,)), int(S["seg_cu"][-1]), d, dtype=dt)
    st["ck"] = N.keys(G, int(S["cu_ctx"][-1]), d, dtype=dt)
    st["mask"] = _dev(S["mask"], np.uint8)[:, None].contiguous()
    st["users"] = (_dev(S["user_off"]), _dev(S["user_req"]))
    # the log-sum-exps that the layer's attention left
    st["lse"] = torch.empty(hq, st["q"].shape[0], device=DEV)
    for b, (q0, tq, *_rest) in enumerate(st["req"]):
        s = _logits(st, b, *_keys_of(st, b))
        st["lse"][:, q0:q0 + tq] = torch.logsumexp(s, -1).reshape(hq, tq)
    for x, like in (("rw", st["rk"]), ("cw", st["ck"])):
        st[x] = torch.zeros(like.shape[:-1], device=DEV)
        st[x + "0"] = N(*like.shape[:-1]).exp_() if case["prior"] else None
    return st


def _prepare_quantize(case, S, N, dt, st):
    G, d = case["hkv"], case["d"]
    if case["kind"] == "pack":
        if case["source"] == "prompt":  # a projection's rows, [tokens][heads][d]
            cu, planes = S["cu_q"], G
            k, v = (N.keys(int(cu[-1]), G, d, dtype=dt).transpose(0, 1), N(int(cu[-1]), G, d, dtype=dt).transpose(0, 1))
        else:
            cu, planes = S["seg_cu"], 1 if case["store"] else G
            k, v = N.keys(planes, int(cu[-1]), d, dtype=dt), N(planes, int(cu[-1]), d, dtype=dt)
        lens = new = np.diff(cu)
        st["len"] = st["cu_new"] = None
        shape = (planes, int(cu[-1]), d)
        codes = [torch.zeros(shape, dtype=torch.uint8, device=DEV).view(F8) for _ in range(2)]
        exps = [torch.zeros(planes, _n_slots(int(cu[-1]), len(cu) - 1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    else:
        cu, lens, new, planes = S["cu_ctx"], S["ctx"], S["q"], G
        st["cu_new"] = st["cu_q"]
        (k8, ke), (v8, ve) = _cache8(N, True, G, cu, lens - new, d), _cache8(N, False, G, cu, lens - new, d)
        codes, exps = [k8, v8], [ke, ve]
        T = int(S["cu_q"][-1])
        # now and then a token that is larger than those before it
        grow = 1 + 3.0 * (torch.rand(T, 1, 1, generator=N.g, device=DEV) > 0.7)
        k = (N.keys(T, G, d) * grow).to(dt).transpose(0, 1)
        v = (N(T, G, d) * grow).to(dt).transpose(0, 1)
    st.update(k=k, v=v, codes=codes, exps=exps, cu=_dev(cu))
    # plain form: new rows and their slots; rows already there in blocks that
    # new ones join; the slots that start with new rows
    row, slot, at = _slots(cu, lens)
    is_new = at >= np.repeat(lens - new, lens)
    joined = np.zeros(_n_slots(int(cu[-1]), len(cu) - 1), bool)
    joined[slot[is_new]] = True
    old = ~is_new & joined[slot]
    held = np.zeros_like(joined)
    held[slot[old]] = True
    st["new"] = (_dev(row[is_new], np.int64), _dev(slot[is_new], np.int64))
    st["old"] = (_dev(row[old], np.int64), _dev(slot[old], np.int64)) if old.any() else None
    st["fresh"] = _dev(joined & ~held, np.bool_)
    return st


# ------------------------------------------------------------------ the plain forms

def _exponent(amax):
    """The smallest e >= 1 with amax <= 448 * 2^(e - 127)."""
    m, x = torch.frexp(amax)
    return torch.where(amax > 0, x + 118 + (m > 0.875), 1).clamp(min=1).to(torch.int32)


def _quantize(x, slot, exps):
    """Codes of rows x[planes][n][d], whose scales are those of `slot`, and the
    exponents: at least exps[planes][slots] and what the rows need."""
    x = x.float()
    x = torch.where(torch.isfinite(x), x, math.nan)
    need = _exponent(torch.nan_to_num(x, nan=0.0).abs().amax(-1))
    exps = exps.scatter_reduce(1, slot.expand(len(x), -1), need, "amax")
    return torch.ldexp(x, 127 - exps[:, slot, None]).to(F8), exps


def _plain_quantize(st):
    row, slot = st["new"]
    for x, codes, exps in ((st["k"], st["codes"][0], st["exps"][0]), (st["v"], st["codes"][1], st["exps"][1])):
        had = exps.to(torch.int32)
        c, e = _quantize(x, slot, torch.where(st["fresh"], 1, had))
        bits = codes.view(torch.uint8)
        if st["old"] is not None:
            row0, slot0 = st["old"]
            c0 = torch.ldexp(bits[:, row0].view(F8).float(), (had - e)[:, slot0, None]).to(F8)
            bits[:, row0] = c0.view(torch.uint8)
        bits[:, row] = c.view(torch.uint8)
        exps.copy_(e)
    return [*st["codes"], *st["exps"]]


def _values(codes, exps, row, slot):
    """float32 values of rows of an 8-bit cache."""
    c = codes.view(torch.uint8).reshape(-1, codes.shape[-1])[row].view(F8).float()
    return torch.ldexp(c, exps.reshape(-1)[slot][..., None].to(torch.int32) - 127)


def _keys_of(st, b, v=False):
    """Request b's resource keys [G][m][d] and context keys [G][tc][d]."""
    _, _, c0, tc, row, slot, _ = st["req"][b]
    x = "v" if v else "k"
    if st["case"]["kind"] == "weigh":
        rk = st["rk"].reshape(-1, st["rk"].shape[-1])
        return rk[row].float(), st["ck"][:, c0:c0 + tc].float()
    c, e = st["c" + x], st["c" + x + "_exp"]
    g = torch.arange(len(c), device=DEV)[:, None]
    ctx = torch.arange(c0, c0 + tc, device=DEV)
    return (_values(st["r" + x], st["r" + x + "_exp"], row, slot),
            _values(c, e, ctx + g * c.shape[1], st["ctx_slot"][b] + g * e.shape[1]))


def _logits(st, b, rk, ck):
    """Scaled logits [G][heads * queries][keys] of request b, -inf where unseen."""
    q0, tq, _, tc, _, _, seen = st["req"][b]
    G, d = len(ck), ck.shape[-1]
    q = st["q"][q0:q0 + tq].to(rk.dtype).permute(1, 0, 2).reshape(G, -1, d)
    k = torch.cat([rk, ck], 1)
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
    m = rk.shape[1]
    s[:, :, :m].masked_fill_(~seen[:, None], -math.inf)
    if tq > 1:
        later = torch.arange(tc, device=DEV)[None] > tc - tq + torch.arange(tq, device=DEV)[:, None]
        s.view(G, -1, tq, m + tc)[..., m:].masked_fill_(later, -math.inf)
    return s


def _plain_attend(st):
    for b, (q0, tq, *_rest) in enumerate(st["req"]):
        s = _logits(st, b, *_keys_of(st, b))
        p = (s - s.amax(-1, keepdim=True)).exp_()
        o = torch.matmul(p, torch.cat(_keys_of(st, b, v=True), 1)) / p.sum(-1, keepdim=True)
        G, d = o.shape[0], o.shape[2]
        st["out"][q0:q0 + tq] = o.view(-1, tq, d).permute(1, 0, 2).to(st["out"].dtype)
    return [st["out"]]


def _plain_weigh(st):
    G = st["case"]["hkv"]
    for x in ("rw", "cw"):
        st[x].copy_(st[x + "0"]) if st[x + "0"] is not None else st[x].zero_()
    for b, (q0, tq, c0, tc, row, _, seen) in enumerate(st["req"]):
        s = _logits(st, b, *_keys_of(st, b))
        w = (s - st["lse"][:, q0:q0 + tq].reshape(G, -1, 1)).exp_().sum(1)
        m = row.shape[1]
        st["rw"].view(-1).index_add_(0, row.reshape(-1), w[:, :m].reshape(-1))
        st["cw"][:, c0:c0 + tc] += w[:, m:]
    return [st["rw"], st["cw"]]


def _plain_evict(st):
    score = st["w"].double().sum(0).float()
    score = torch.where(st["forced"], math.inf, score)
    # best first within every segment, equal scores in their order
    order = torch.sort(score, descending=True, stable=True).indices
    order = order[torch.sort(st["seg"][order], stable=True).indices]
    place = torch.empty_like(order)
    place[order] = torch.arange(len(order), device=DEV)
    cu = st["cu"].long()
    k = (st["cu_kept"][1:] - st["cu_kept"][:-1]).long()
    kept = torch.nonzero(place - cu[st["seg"]] < k[st["seg"]])[:, 0]
    st["kept"].copy_(kept - cu[st["seg"][kept]])
    st["kept_w"].copy_(st["w"][:, kept])
    return [st["kept"], st["kept_w"]]


# ------------------------------------------------------------------ run

def run(st):
    case, kind = st["case"], st["case"]["kind"]
    if not own:
        return {"pack": _plain_quantize, "append": _plain_quantize, "attend": _plain_attend,
                "weigh": _plain_weigh, "evict": _plain_evict}[kind](st)
    from paper_2608_19662_amd import recache as rc
    if kind in ("pack", "append"):
        rc.quantize_kv(st["k"], st["v"], *st["codes"], *st["exps"], st["cu"], lens=st["len"], cu_new=st["cu_new"])
        return [*st["codes"], *st["exps"]]
    if kind == "evict":
        ws = st["ws"].get("ws")
        if ws is None:  # a program keeps it from call to call
            nb = rc.select_workspace_bytes(len(st["cu"]) - 1, st["w"].shape[1], st["max_len"])
            ws = st["ws"]["ws"] = torch.empty(max(nb, 1), dtype=torch.uint8, device=DEV)
        rc.select_kept(st["w"], st["cu"], st["cu_kept"], st["kept"], max_len=st["max_len"], kept_w=st["kept_w"],
                       keep_first=case["first"], keep_last=case["last"], workspace=ws)
        return [st["kept"], st["kept_w"]]
    if kind == "weigh":
        rc.attend_weights(st["q"], st["lse"], st["cu_q"], st["cu_ctx"], st["max_q"], st["cu_kept"], st["mask"],
                          *st["users"], 0, ctx_k=st["ck"], ctx_w=st["cw"], ctx_w_prior=st["cw0"], res_k=st["rk"],
                          res_w=st["rw"], res_w_prior=st["rw0"], res_off=st["res_off"])
        return [st["rw"], st["cw"]]
    route_off, route_res, route_tokens = st["route"]
    rc.attend_quantized(st["q"], st["ck"], st["cv"], st["ck_exp"], st["cv_exp"], st["cu_q"], st["cu_ctx"], st["max_q"],
                        st["max_ctx"], st["rk"], st["rv"], st["rk_exp"], st["rv_exp"], st["cu_kept"], route_off,
                        route_res, route_tokens.view(-1), 0, 1, st["out"], ctx_len=st["len"],
                        max_route_len=case["per_req"], max_kv=st["max_kv"], workspace=st["ws"], res_off=st["res_off"])
    return [st["out"]]


# ------------------------------------------------------------------ work

def work(case):
    if case["kind"] == "evict":
        S = _evict_structure(case)
        return {"bytes": 4.0 * (case["planes"] * (S["cu"][-1] + S["cu_kept"][-1]) + S["cu_kept"][-1]), "flops": 0.0}
    S, G, d = _structure(case), case["hkv"], case["d"]
    wide = d * (4 if case["dtype"] == "f32" else 2)
    if case["kind"] in ("pack", "append"):
        if case["kind"] == "append":
            rows = float(S["q"].sum()) * G
        else:
            rows = float(S["cu_q"][-1]) * G if case["source"] == "prompt" else float(S["seg_cu"][-1]) * (1 if case["store"] else G)
        return {"bytes": 2 * rows * (wide + d + 1 / BLOCK), "flops": 0.0}
    q, ctx = S["q"].astype(np.float64), S["ctx"].astype(np.float64)
    pairs = float((q[:, None] * S["vis"]).sum() + (q * (q + 1) / 2 + q * (ctx - q)).sum() * G) * (case["hq"] // G)
    rows = S["rows"][:, None] * S["mask"]  # of the resources that a request lists
    rows = float(rows[np.unique(S["lists"])].sum()) + float(ctx.sum()) * G
    if case["kind"] == "weigh":
        return {"bytes": rows * (wide + 4 * (1 + case["prior"])) + q.sum() * case["hq"] * (wide + 4), "flops": 2.0 * d * pairs}
    return {"bytes": 2 * rows * (d + 1 / BLOCK) + 2 * q.sum() * case["hq"] * wide, "flops": 4.0 * d * pairs}


# ------------------------------------------------------------------ in 64 bits

def _round_e4m3(y):
    """Nearest e4m3 value (ties to even) of |y| <= 448, in 64 bits."""
    a = y.abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    r = torch.round(a / step) * step
    return torch.where(y < 0, -r, r)


def _exact_quantize(st):
    got, whole = [], []
    new, slot = (t.cpu().numpy() for t in st["new"])
    fresh = st["fresh"]
    for x, codes, exps in zip((st["k"], st["v"]), st["codes"], st["exps"]):
        x, val = x.double(), codes.float().double()
        had = exps.double()
        amax = torch.zeros_like(had).scatter_reduce(1, st["new"][1].expand(len(x), -1), x.abs().amax(-1), "amax")
        need = torch.where(amax > 0, torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448)) + 127, 1).clamp(min=1)
        # (a logarithm next to a whole number is put right by the definition)
        need = need - ((need > 1) & (amax <= 448 * torch.exp2(need - 128))).double()
        need = need + (amax > 448 * torch.exp2(need - 127)).double()
        touched = torch.zeros_like(fresh)
        touched[st["new"][1]] = True
        e = torch.where(touched, torch.maximum(need, torch.where(fresh, 1.0, had)), had)
        if st["old"] is not None:
            r, s = st["old"]
            val[:, r] = _round_e4m3(val[:, r] * torch.exp2(had - e)[:, s, None])
        r, s = st["new"]
        val[:, r] = _round_e4m3(x * torch.exp2(127 - e)[:, s, None])
        got.append(val)
        whole.append(e.to(torch.uint8))
    return got + whole


def _exact_rows(st, name):
    """A cache of an attend case in 64 bits, [planes * rows][d]."""
    return st[name].view(torch.uint8).reshape(-1, st[name].shape[-1])


def _exact_side(st, b, side, x):
    """Keys ("k") or values ("v") of request b, resource or context, in 64 bits."""
    _, _, c0, tc, row, slot, _ = st["req"][b]
    codes, exps = st[side + x], st.get(side + x + "_exp")
    if side == "c":
        p = torch.arange(codes.shape[0], device=DEV)[:, None]
        row = p * codes.shape[1] + torch.arange(c0, c0 + tc, device=DEV)
        slot = None if exps is None else p * exps.shape[1] + st["ctx_slot"][b]
    if exps is None:
        return codes.reshape(-1, codes.shape[-1])[row].double()
    c = _exact_rows(st, side + x)[row].view(F8).to(torch.float32).double()
    return c * torch.exp2(exps.reshape(-1)[slot].double() - 127)[..., None]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("pack", "append"):
        return _exact_quantize(st)
    if kind == "evict":
        S = _evict_structure(case)
        w = st["w"].cpu().numpy()
        score = w.astype(np.float64).sum(0).astype(np.float32).astype(np.float64)
        score[st["forced"].cpu().numpy()] = np.inf
        kept = []
        for s in range(len(S["len"])):
            z = score[S["cu"][s]:S["cu"][s + 1]]
            kept.append(np.sort(np.argsort(-z, kind="stable")[:S["k"][s]]) + S["cu"][s])
        at = np.concatenate(kept)
        return [torch.from_numpy((at - np.repeat(S["cu"][:-1], S["k"])).astype(np.int32)),
                torch.from_numpy(w[:, at].astype(np.float64))]
    G, d = case["hkv"], case["d"]
    if kind == "attend":
        out = torch.empty(st["q"].shape, dtype=torch.float64, device=DEV)
    else:
        rw = torch.zeros(st["rw"].shape, dtype=torch.float64, device=DEV) if st["rw0"] is None else st["rw0"].double()
        cw = torch.zeros(st["cw"].shape, dtype=torch.float64, device=DEV) if st["cw0"] is None else st["cw0"].double()
    for b, (q0, tq, c0, tc, row, _, seen) in enumerate(st["req"]):
        k = torch.cat([_exact_side(st, b, "r", "k"), _exact_side(st, b, "c", "k")], 1)
        v = torch.cat([_exact_side(st, b, "r", "v"), _exact_side(st, b, "c", "v")], 1) if kind == "attend" else None
        m = row.shape[1]
        R = case["hq"] // G
        for g in range(G):
            sum_w = torch.zeros(m + tc, dtype=torch.float64, device=DEV)
            for i0 in range(0, tq, 512):
                i1 = min(tq, i0 + 512)
                q = st["q"][q0 + i0:q0 + i1, g * R:(g + 1) * R].double().reshape(-1, d)
                z = (q @ k[g].t().contiguous() / math.sqrt(d)).view(i1 - i0, R, -1)
                ok = torch.cat([seen[g][None].expand(i1 - i0, -1), torch.arange(tc, device=DEV)[None] <=
                                tc - tq + torch.arange(i0, i1, device=DEV)[:, None]], 1)
                z = z.masked_fill(~ok[:, None], -math.inf)
                if kind == "attend":
                    o = torch.softmax(z, -1).view(-1, m + tc) @ v[g]
                    out[q0 + i0:q0 + i1, g * R:(g + 1) * R] = o.view(i1 - i0, R, d)
                else:
                    l = st["lse"][g * R:(g + 1) * R, q0 + i0:q0 + i1].double().t()
                    sum_w += (z - l[..., None]).exp().sum((0, 1))
            if kind == "weigh":
                flat = rw.view(-1)
                flat[row[g][seen[g]]] += sum_w[:m][seen[g]]
                cw[g, c0:c0 + tc] += sum_w[m:]
    return [out] if kind == "attend" else [rw, cw]
