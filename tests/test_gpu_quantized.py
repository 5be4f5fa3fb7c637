"""8-bit caches on the GPU: quantize_kv bit for bit against its definition, and
attend_quantized against attention in 64 bits over the caches' values.

Tolerance of an attention output (everything else is exact).  A code times its
scale is exact in bf16, so the operands of both sides are the same.  What the
kernels round: the weights of the P V product to bf16 (half a step, 2^-8 of each;
the row sum is of the rounded ones, so that the output moves by at most
2^-8 / (1 - 2^-8) of the weighted mean distance of the values from it), the
output to bf16 (2^-8 of it), and in fp32 the logits, exponentials and sums: a logit
is a sum of d products whose absolute values sum to at most A, off by at most d
2^-24 A, its multiple of log2(e) and the difference to the reference by 2^-23 |s| each,
which moves every weight by that; sums of n weights or products by n 2^-24.
With d <= 128, A <= 40, |s| <= 40, n <= 5000: under 7e-4 of the mean distance and
of the output's own sum of absolute terms (at most spread + |out|).  So
    |gpu - ref| <= (2^-8 * 1.005 + 7e-4) spread + (2^-8 + 7e-4) |ref| + 1e-6
LSE: the row sum is of rounded weights, so within ln(1 + 2^-8) + 7e-4 of the exact one."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from gpu_helpers import DEV, Routes, f64, i32
from paper_2608_19662_amd import recache as rc
from paper_2608_19662_amd.workloads import AttendWorkload, prefix
from test_gpu_parity import small_attend

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def u8(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def bits(t):
    return t.view(torch.uint8).cpu().numpy()


# ------------------------------------------------------------------- quantize_kv

def source(rng, shape, dtype):
    """Rows of very different size, exact zeros among them, and values on the
    borders of a scale."""
    x = rng.normal(size=shape) * np.exp(3 * rng.normal(size=shape[:-1] + (1,)))
    x[..., ::7, :] *= 0
    x[..., 3, 5] = 1.75 * 2.0 ** rng.integers(-3, 4)
    x[..., -1, 0] = 1.7578125 * 2.0 ** rng.integers(-3, 4)
    t = torch.from_numpy(x).to(dtype)
    return t


def run_quantize(cu, rows, planes, d, dtype, layout, lens=None, cu_new=None, seed=1, before=None, stream=None):
    """(GPU, reference) codes and exponents of K and V, from `before` (codes, exps of both)."""
    rng = np.random.default_rng(seed)
    src = rows if cu_new is None else int(cu_new[-1])
    blocks = rc.quantized_blocks(rows, len(cu) - 1)
    if before is None:
        before = [(np.full((planes, rows, d), 0x35, np.uint8), np.full((planes, blocks), 99, np.uint8)) for _ in "kv"]
    xs = [source(rng, (planes, max(src, 8), d), dtype)[:, :src].contiguous() for _ in "kv"]
    dev = []
    for x in xs:
        if layout == "heads":      # [planes][rows][d]
            dev.append(x.to(DEV))
        elif layout == "tokens":   # [rows][planes][d]
            dev.append(x.transpose(0, 1).contiguous().to(DEV).transpose(0, 1))
        else:                      # a slice of a fused projection, rows of more heads and planes than these
            wide = torch.zeros(src + 3, planes + 2, d, dtype=dtype)
            wide[1:src + 1, 1:planes + 1] = x.transpose(0, 1)
            dev.append(wide.to(DEV)[1:src + 1, 1:planes + 1].transpose(0, 1))
    k8, v8 = (u8(b[0]).view(F8) for b in before)
    ke, ve = (u8(b[1]) for b in before)
    rc.quantize_kv(*dev, k8, v8, ke, ve, i32(cu), lens=None if lens is None else i32(lens),
                   cu_new=None if cu_new is None else i32(cu_new), stream=stream)
    torch.cuda.synchronize()
    want = []
    for x, (c, e) in zip(xs, before):
        c, e = c.copy(), e.copy()
        ref.quantize(x.double().numpy(), c, e, cu, lens, cu_new)
        want.append((c, e))
    return [(bits(k8), bits(ke)), (bits(v8), bits(ve))], want


def assert_same(got, want, what=""):
    for (gc, ge), (wc, we), name in zip(got, want, "kv"):
        assert np.array_equal(ge, we), (what, name, "exponents", np.argwhere(ge != we)[:4])
        # +0 and -0 are both right where a value rounds to nothing
        g, w = ref.VALUES[gc], ref.VALUES[wc]
        same = (gc == wc) | ((g == 0) & (w == 0)) | (np.isnan(g) & np.isnan(w))
        assert same.all(), (what, name, "codes", np.argwhere(~same)[:4])


LENGTHS = [1, 63, 64, 65, 0, 127, 128, 129, 300, 2, 0, 17]


@pytest.mark.parametrize("layout", ["heads", "tokens", "slice"])
@pytest.mark.parametrize("planes,d,dtype", [(8, 128, torch.bfloat16), (1, 128, torch.float32), (3, 64, torch.bfloat16),
                                            (2, 64, torch.float32)])
def test_quantize_all_rows(planes, d, dtype, layout):
    cu = prefix(LENGTHS)
    assert_same(*run_quantize(cu, int(cu[-1]), planes, d, dtype, layout))


def test_quantize_one_row_and_many_segments():
    assert_same(*run_quantize(prefix([1]), 1, 1, 128, torch.bfloat16, "heads"))
    rng = np.random.default_rng(4)
    cu = prefix(rng.integers(0, 4, 5000))  # more than two steps of the segment search
    assert_same(*run_quantize(cu, int(cu[-1]), 2, 64, torch.bfloat16, "heads"))


def test_quantize_segments_with_room():
    """Rows and scales past each segment's length stay as they are."""
    cap = [100, 64, 200, 65, 1]
    lens = np.array([70, 64, 0, 1, 1])
    cu = prefix(cap)
    got, want = run_quantize(cu, int(cu[-1]) + 30, 2, 128, torch.bfloat16, "heads", lens=lens)
    assert_same(got, want)
    assert (got[0][0][:, 70:100] == 0x35).all() and (got[0][0][:, int(cu[-1]):] == 0x35).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_quantize_appends(dtype, layout):
    """New rows join blocks that hold rows already, in one call and token by token."""
    cap = [200, 64, 300, 130, 70, 65]
    cu = prefix(cap)
    rng = np.random.default_rng(7)
    lens = np.array([60, 0, 64, 100, 1, 63])
    state = run_quantize(cu, int(cu[-1]), 2, 128, dtype, layout, lens=lens, seed=11)
    assert_same(*state)
    for step in range(6):
        new = rng.integers(0, 5, 6) if step % 2 else np.array([1, 1, 1, 1, 1, 1])
        if step == 4:
            new[2] = 130
        new = np.minimum(new, np.array(cap) - lens)
        lens = lens + new
        state = run_quantize(cu, int(cu[-1]), 2, 128, dtype, layout, lens=lens, cu_new=prefix(new), seed=20 + step,
                             before=state[1])
        assert_same(*state, what=step)


@pytest.mark.parametrize("dtype,d,planes,rows", [(torch.bfloat16, 128, 8, 90_000), (torch.float32, 64, 5, 180_001)])
def test_quantize_many_rows(dtype, d, planes, rows):
    """More than twice the last-level cache in one call, and plane by plane."""
    g = torch.Generator(device=DEV).manual_seed(17)
    k, v = (torch.randn(rows, planes, d, generator=g, device=DEV).to(dtype).transpose(0, 1) for _ in "kv")
    assert k.numel() * 2 * (k.element_size() + 1) >= 512 << 20
    cu = i32([0, 7, 7, rows // 2, rows])
    blocks = rc.quantized_blocks(rows, 4)
    one, many = ([torch.zeros(planes, rows, d, dtype=torch.uint8, device=DEV) for _ in "kv"]
                 + [torch.zeros(planes, blocks, dtype=torch.uint8, device=DEV) for _ in "kv"] for _ in range(2))
    rc.quantize_kv(k, v, *one, cu)
    for p in range(planes):
        rc.quantize_kv(k[p:p + 1], v[p:p + 1], *[t[p:p + 1] for t in many], cu)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(one, many))
    n = 300  # and by the definition at the end
    c, e = np.zeros((1, rows - rows // 2, d), np.uint8), np.zeros((1, blocks), np.uint8)
    ref.quantize(v[-1:, rows // 2:].cpu().double().numpy(), c, e, np.array([0, rows - rows // 2]))
    assert np.array_equal(bits(one[1])[-1, -n:], c[0, -n:])


def test_quantize_values_that_are_not_finite():
    x = np.random.default_rng(3).normal(size=(1, 130, 128))
    x[0, 3, 4], x[0, 5, 6], x[0, 66, 0] = np.inf, np.nan, -np.inf
    x[0, 129] = np.nan  # a block without any finite value
    cu = [0, 129, 130]
    k = torch.from_numpy(x).to(torch.bfloat16).to(DEV)
    blocks = rc.quantized_blocks(130, 2)
    k8, v8 = (torch.zeros(1, 130, 128, dtype=torch.uint8, device=DEV) for _ in "kv")
    ke, ve = (torch.zeros(1, blocks, dtype=torch.uint8, device=DEV) for _ in "kv")
    rc.quantize_kv(k, k, k8, v8, ke, ve, i32(cu))
    torch.cuda.synchronize()
    c, e = np.zeros((1, 130, 128), np.uint8), np.zeros((1, blocks), np.uint8)
    ref.quantize(k.cpu().double().numpy(), c, e, cu)
    assert_same([(bits(k8), bits(ke)), (bits(v8), bits(ve))], [(c, e), (c, e)])
    assert np.isnan(ref.VALUES[bits(k8)[0, 3, 4]]) and np.isnan(ref.VALUES[bits(k8)[0, 129]]).all()


def test_quantize_every_bf16_value():
    """Each finite bf16 at each of several scales of its block."""
    v = np.arange(65536, dtype=np.uint16).view(np.int16)
    t = torch.from_numpy(v).view(torch.bfloat16)
    t = t[torch.isfinite(t.float())]
    n = t.numel() // 126 * 126
    for big in (0.0, 448.0, 2.0 ** 60, 3e38):
        x = torch.zeros(1, n // 126, 128, dtype=torch.bfloat16)
        x[0, :, :126] = t[:n].view(-1, 126)
        x[0, :, 127] = big
        # a block per row
        cu = np.arange(n // 126 + 1)
        k8, v8 = (torch.zeros(x.shape, dtype=torch.uint8, device=DEV) for _ in "kv")
        blocks = rc.quantized_blocks(n // 126, n // 126)
        ke, ve = (torch.zeros(1, blocks, dtype=torch.uint8, device=DEV) for _ in "kv")
        rc.quantize_kv(x.to(DEV), x.to(DEV), k8, v8, ke, ve, i32(cu))
        torch.cuda.synchronize()
        c, e = np.zeros(x.shape, np.uint8), np.zeros((1, blocks), np.uint8)
        ref.quantize(x.double().numpy(), c, e, cu)
        assert_same([(bits(k8), bits(ke)), (bits(v8), bits(ve))], [(c, e), (c, e)], what=big)


# -------------------------------------------------------------- attend_quantized

def check_attend(out, lse, want, what):
    o, l, spread = want
    bound = (2.0 ** -8 * 1.005 + 7e-4) * spread + (2.0 ** -8 + 7e-4) * np.abs(o) + 1e-6
    err = np.abs(f64(out) - o)
    assert (err <= bound).all(), (what, float(err.max()), float((err / bound).max()), np.argwhere(~(err <= bound))[:3])
    if lse is not None:
        err = np.abs(f64(lse) - l)
        assert (err <= np.log1p(2.0 ** -8) + 7e-4).all(), (what, "lse", float(err.max()))


def pack(x, cu, lens=None):
    """Codes and exponents of one tensor [planes][rows][d] by the library, and their values in 64 bits."""
    blocks = rc.quantized_blocks(x.shape[1], len(cu) - 1)
    # what no row touches holds NaN codes and large scales
    c = [torch.full(x.shape, 0x7F, dtype=torch.uint8, device=DEV) for _ in "kv"]
    e = [torch.full((x.shape[0], blocks), 240, dtype=torch.uint8, device=DEV) for _ in "kv"]
    rc.quantize_kv(x, x, *c, *e, i32(cu), lens=None if lens is None else i32(lens))
    torch.cuda.synchronize()
    return c[0].view(F8), e[0], ref.dequantize(bits(c[0]), bits(e[0]), cu, lens)


class Packed:
    """An AttendWorkload's layer in 8 bits: per-head caches or a route-compacted
    store, contexts packed or with room to grow."""

    def __init__(self, w, layer, store=False, slack=0, scale=1.0):
        self.w, self.layer, self.store = w, layer, store
        q, ck, cv, rk, rv = w.layer_tensors(layer, DEV)
        self.q = (q.float() * scale).to(torch.bfloat16)
        self.rt = Routes(w)
        # contexts: room of `slack` rows behind each
        self.ctx_off = prefix(np.asarray(w.ctx_lens) + slack)
        if slack:
            wide = [torch.full((w.n_kv_heads, int(self.ctx_off[-1]), w.head_dim), float("nan"), dtype=t.dtype,
                               device=DEV) for t in (ck, cv)]
            for x, t in zip(wide, (ck, cv)):
                for b in range(w.n_req):
                    x[:, self.ctx_off[b]:self.ctx_off[b] + w.ctx_lens[b]] = t[:, w.cu_ctx[b]:w.cu_ctx[b + 1]]
            ck, cv = wide
        lens = w.ctx_lens if slack else None
        self.ck, self.cke, self.ck64 = pack(ck, self.ctx_off, lens)
        self.cv, self.cve, self.cv64 = pack(cv, self.ctx_off, lens)
        self.ctx_len = i32(w.ctx_lens) if slack else None
        self.seg_off = self.res_off = None
        if store:
            off = self.rt.store_offsets()[layer]
            self.seg_off, self.res_off = off.cpu().numpy(), off
            rows = int(self.seg_off[-1])
            ks, vs = (torch.zeros(rows, w.head_dim, dtype=rk.dtype, device=DEV) for _ in "kv")
            K = int(w.cu_rows[-1])
            rc.store_routes(rk, rv, self.rt.cu_rows, self.rt.cu_rows,
                            i32(np.concatenate([np.arange(n) for n in np.diff(w.cu_rows)])), self.rt.store_offsets(),
                            layer, ks, vs, total_kept=K)
            (self.rk, self.rke, k64), (self.rv, self.rve, v64) = pack(ks[None], self.seg_off), pack(vs[None], self.seg_off)
            self.rk, self.rv, self.rke, self.rve = self.rk[0], self.rv[0], self.rke[0], self.rve[0]
            self.rk64, self.rv64 = k64[0], v64[0]
        else:
            self.rk, self.rke, self.rk64 = pack(rk, w.cu_rows)
            self.rv, self.rve, self.rv64 = pack(rv, w.cu_rows)
        self.mkv = self.rt.max_kv(layer)

    def workspace(self):
        return self.rt.workspace(self.mkv)

    def run(self, lse=True, plan=None, stream=None, workspace=None, max_kv=None, out=None, softmax_scale=0.0):
        w, rt = self.w, self.rt
        out = torch.full_like(self.q, float("nan")) if out is None else out
        l = torch.full((w.n_q_heads, self.q.shape[0]), float("nan"), device=DEV) if lse else None
        rc.attend_quantized(self.q, self.ck, self.cv, self.cke, self.cve, rt.cu_q, i32(self.ctx_off), rt.max_q, rt.max_ctx,
                            self.rk, self.rv, self.rke, self.rve, rt.cu_rows, rt.route_off, rt.route_res,
                            rt.route_tokens, self.layer, w.n_layers, out, ctx_len=self.ctx_len,
                            max_route_len=max(rt.max_route_len, 1), lse=l,
                            workspace=self.workspace() if workspace is None else workspace,
                            max_kv=self.mkv if max_kv is None else max_kv, softmax_scale=softmax_scale,
                            res_off=self.res_off, plan=plan, stream=stream)
        return out, l

    def want(self, scale=None):
        return ref.attend(self.w, self.q.cpu().double().numpy(), self.rk64, self.rv64, self.ck64, self.cv64, self.layer,
                          scale=scale, seg_off=self.seg_off, ctx_off=self.ctx_off)


HEADS = [(32, 8, 128), (8, 2, 64), (28, 4, 128), (8, 8, 128), (16, 2, 64), (12, 4, 64), (4, 2, 128)]


@pytest.mark.parametrize("store,slack", [(False, 0), (True, 0), (False, 37), (True, 130)])
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_attend_decode(Hq, Hkv, d, store, slack):
    w = small_attend(31 + Hq, 6, 9, Hq, Hkv, d, "bf16", [1] * 6, [1, 63, 64, 65, 700, 129], max_len=500)
    p = Packed(w, 1, store, slack)
    out, lse = p.run()
    check_attend(out, lse, p.want(), "decode")
    out2, lse2 = p.run(plan=p.rt.plan())
    out3, _ = p.run(lse=False)
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(out, out3)


@pytest.mark.parametrize("store,slack", [(False, 0), (True, 0), (False, 37), (True, 130)])
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_attend_prefill(Hq, Hkv, d, store, slack):
    w = small_attend(57 + Hq, 5, 9, Hq, Hkv, d, "bf16", [1, 33, 64, 2, 70], [1, 33, 130, 65, 200], max_len=400)
    p = Packed(w, 2, store, slack)
    out, lse = p.run()
    check_attend(out, lse, p.want(), "prefill")
    out2, lse2 = p.run(plan=p.rt.plan())
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("Hq,Hkv,d,q,ctx", [
    (32, 8, 128, [150] * 6, [150, 400, 151, 200, 150, 300]),    # a full grid
    (8, 1, 64, [300, 1, 5], [320, 900, 6]),
    (64, 8, 128, [40] * 20, [41] * 20),
])
def test_attend_prefill_grids(Hq, Hkv, d, q, ctx):
    w = small_attend(77, len(q), 6, Hq, Hkv, d, "bf16", q, ctx, max_len=200)
    p = Packed(w, 0)
    out, lse = p.run()
    check_attend(out, lse, p.want(), "grid")


@pytest.mark.parametrize("Hq,Hkv,d,q,ctx,store,slack", [
    (32, 8, 128, [150] * 11 + [7], [150 + 37 * i for i in range(11)] + [500], False, 0),
    (16, 2, 64, [470] * 7 + [1, 33], [470, 471, 500, 534, 600, 480, 512, 700, 40], True, 19),
    (64, 8, 128, [1 + i % 9 for i in range(210)], [9 + i for i in range(210)], False, 0),  # many small requests
])
def test_attend_prefill_grids_of_blocks(Hq, Hkv, d, q, ctx, store, slack):
    """More than 1,600 blocks of 32 columns."""
    w = small_attend(78, len(q), 6, Hq, Hkv, d, "bf16", q, ctx, max_len=200)
    p = Packed(w, 0, store, slack)
    out, lse = p.run()
    check_attend(out, lse, p.want(), "grid of blocks")
    out2, lse2 = p.run(plan=p.rt.plan())
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("Hq,Hkv,d,n", [(32, 8, 128, 11), (8, 8, 64, 44), (32, 8, 128, 2), (8, 8, 64, 4)])
def test_attend_prefill_queries_of_uneven_size(Hq, Hkv, d, n):
    """Dims of very different size within a query, large grids and small.
    Queries may be taken in parts that are off by up to 2^-21 of the largest of their 64 dims:
    a logit by delta = scale 2^-21 sum over those 64 of (that largest * sum |k|), every
    weight by it, the output by at most 2 delta of the mean distance."""
    w = small_attend(79, n, 6, Hq, Hkv, d, "bf16", [150] * n, [150 + 17 * i for i in range(n)], max_len=200)
    p = Packed(w, 0)
    size = torch.ones(d, device=DEV)
    size[:32], size[32:64] = 2.0 ** -9, 1.5
    size[d - 7] = 6.0
    size[d - 3], size[5] = 2.0 ** -12, 2.0 ** -20
    p.q = (p.q.float() * size).to(torch.bfloat16)
    out, lse = p.run()
    o, l, spread = p.want()
    qmax = p.q.float().abs().view(-1, Hq, d // 64, 64).amax(-1).amax((0, 1)).cpu().numpy()
    ksum = max(np.abs(x).reshape(-1, d // 64, 64).sum(-1)[np.isfinite(x).reshape(-1, d).all(-1)].max(0).dot(qmax)
               for x in (p.rk64, p.ck64))
    delta = ksum * 2.0 ** -21 / np.sqrt(d)
    assert delta < 1e-3
    err = np.abs(f64(out) - o)
    bound = (2.0 ** -8 * 1.005 + 7e-4 + 2 * delta) * spread + (2.0 ** -8 + 7e-4) * np.abs(o) + 1e-6
    assert (err <= bound).all(), float((err / bound).max())
    assert (np.abs(f64(lse) - l) <= np.log1p(2.0 ** -8) + 7e-4 + delta).all()


@pytest.mark.parametrize("q", [1, 40])
def test_attend_without_resources(q):
    """No request lists anything; no resource rows at all."""
    w = AttendWorkload(seed=3, n_layers=1, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype="bf16",
                       lengths=np.array([5], np.int32), req_res_off=np.array([0, 0, 0], np.int32),
                       req_res=np.zeros(0, np.int32), q_lens=np.array([q, q], np.int32),
                       ctx_lens=np.array([q, 90], np.int32), mask=np.ones((1, 1, 2), np.uint8))
    p = Packed(w, 0)
    out, lse = p.run()
    check_attend(out, lse, p.want(), "no resources")


@pytest.mark.parametrize("q", [1, 3])
def test_attend_many_resources(q):
    """Route lists of 1024 resources of one to five rows, past it NaN."""
    n = 1025
    rng = np.random.default_rng(5)
    lengths = rng.integers(1, 6, n).astype(np.int32)
    lists = [np.arange(1024), rng.permutation(n)[:700], np.arange(1025)]
    w = AttendWorkload(seed=6, n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="bf16", lengths=lengths,
                       req_res_off=prefix([len(x) for x in lists]), req_res=np.concatenate(lists).astype(np.int32),
                       q_lens=np.array([q] * 3, np.int32), ctx_lens=np.array([q, 70, q], np.int32),
                       mask=np.ones((n, 1, 2), np.uint8))
    p = Packed(w, 0)
    p.rt.max_route_len = 1024
    out, lse = p.run()
    torch.cuda.synchronize()
    assert torch.isnan(out[2 * q:].float()).all()
    o, l, s = p.want()
    check_attend(out[:2 * q], lse[:, :2 * q], (o[:2 * q], l[:, :2 * q], s[:2 * q]), "1024 resources")


@pytest.mark.parametrize("q", [1, 50])
def test_attend_rising_logits(q):
    """Logits of hundreds, rising along the stream: the reference max moves."""
    w = small_attend(91, 3, 5, 8, 2, 128, "bf16", [q] * 3, [q + 5, 300, 500], max_len=300, mask_p=1.0)
    p = Packed(w, 0, scale=1.0)
    # keys grow along every segment
    k64 = []
    for t, cu in ((w.layer_tensors(0, DEV)[3], w.cu_rows), (w.layer_tensors(0, DEV)[1], w.cu_ctx)):
        at = torch.cat([torch.arange(int(cu[i + 1] - cu[i])) for i in range(len(cu) - 1)]).to(DEV)
        k64.append(pack((t.float() * (1 + at[None, :, None] / 40.0)).to(torch.bfloat16), cu))
    (p.rk, p.rke, p.rk64), (p.ck, p.cke, p.ck64) = k64
    out, lse = p.run()
    o, l, spread = p.want()
    # |s| reaches 100 here and A 300: the fp32 terms are up to 128 * 2^-24 * 300 + 3 * 2^-23 * 100 < 2.4e-3
    bound = (2.0 ** -8 * 1.005 + 3e-3) * spread + (2.0 ** -8 + 3e-3) * np.abs(o) + 1e-6
    assert (np.abs(f64(out) - o) <= bound).all()
    assert (np.abs(f64(lse) - l) <= np.log1p(2.0 ** -8) + 3e-3).all()


@pytest.mark.parametrize("q", [1, 20])
def test_attend_nan_reaches_those_who_see_it(q):
    """A NaN row of a resource spoils the requests that see it and no others; one
    in a later context row only the rows from there on."""
    w = small_attend(19, 3, 3, 8, 2, 128, "bf16", [q] * 3, [q + 30] * 3, max_len=200, mask_p=1.0)
    w.req_res_off, w.req_res = prefix([2, 1, 1]), np.array([0, 2, 1, 2], np.int32)
    p = Packed(w, 0)
    p.rv.view(torch.uint8)[0, int(w.cu_rows[1]) - 1, 7] = 0x7F  # the last row of resource 0, group 0
    out, _ = p.run()
    torch.cuda.synchronize()
    bad = torch.isnan(out.float())
    assert bad[:q, :4, 7].all() and int(bad.sum()) == q * 4
    p.ck.view(torch.uint8)[1, int(p.ctx_off[2]) + 30 + q - 1, 0] = 0x7F  # the newest key of request 2, group 1
    out, _ = p.run()
    torch.cuda.synchronize()
    bad = torch.isnan(out[2 * q:].float()).flatten(1).any(1)
    assert bad[-1] and int(bad.sum()) == 1


def test_attend_is_the_16_bit_call_on_the_values():
    """attend_cached over the caches' values in bf16, which hold them exactly."""
    for q in ([1] * 4, [40, 3, 129, 64]):
        w = small_attend(23, 4, 8, 32, 8, 128, "bf16", q, [300, 77, 200, 64], max_len=400)
        p = Packed(w, 1)
        out, lse = p.run()
        bf = [torch.from_numpy(x).to(torch.bfloat16).to(DEV) for x in (p.ck64, p.cv64, p.rk64, p.rv64)]
        for x, y in zip(bf, (p.ck64, p.cv64, p.rk64, p.rv64)):
            assert np.array_equal(f64(x), y)
        o2, l2 = p.rt.attend(p.q, *bf, 1, workspace=p.workspace(), max_kv=p.mkv)
        torch.cuda.synchronize()
        want = p.want()
        check_attend(o2, l2, want, "attend_cached")
        check_attend(out, lse, want, "attend_quantized")


def test_attend_scale_and_repeat():
    w = small_attend(29, 3, 5, 16, 4, 128, "bf16", [9, 1, 33], [20, 40, 33])
    p = Packed(w, 0)
    out, lse = p.run(softmax_scale=0.25)
    check_attend(out, lse, p.want(scale=0.25), "scale")
    for _ in range(3):
        o, l = p.run(softmax_scale=0.25)
        assert torch.equal(o, out) and torch.equal(l, lse)


def test_attend_sizes_that_understate():
    """More queries than max_q says, and a request of two queries in decode: NaN."""
    w = small_attend(37, 2, 3, 4, 2, 64, "bf16", [40, 70], [50, 80])
    p = Packed(w, 0)
    o, l, s = p.want()
    p.rt.max_q = 64  # total_q <= n_req * max_q still holds
    out, lse = p.run()
    torch.cuda.synchronize()
    assert torch.isnan(out[40 + 64:].float()).all()
    check_attend(out[:104], lse[:, :104], (o[:104], l[:, :104], s[:104]), "understated")


@pytest.mark.parametrize("d", [64, 128])
def test_attend_large_context_planes(d):
    """Contexts that may reach 512 MiB: the rows of the same short ones, at the
    start of large planes, give the same bits."""
    w = small_attend(43, 4, 5, 8, 2, d, "bf16", [1] * 4, [1, 200, 64, 333], max_len=200)
    p = Packed(w, 0)
    out, lse = p.run()
    check_attend(out, lse, p.want(), "short planes")
    rows = (512 << 20) // (2 * d * 2)
    more = rc.quantized_blocks(rows, 4) - p.cke.shape[1]
    grow = lambda t, n, x: torch.cat([t.view(torch.uint8), torch.full((2, n) + t.shape[2:], x, dtype=torch.uint8, device=DEV)], 1)
    p.ck, p.cv = (grow(t, rows - t.shape[1], 0x7F).view(F8) for t in (p.ck, p.cv))
    p.cke, p.cve = (grow(t, more, 240) for t in (p.cke, p.cve))
    p.rt.max_ctx = rows // 4
    out2, lse2 = p.run()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_attend_plane_past_4_gib():
    """A context plane of 4.3 GB per K and V, its last rows in use: offsets pass 32 bits."""
    d, rows, n = 128, 34_000_000, 200
    free = torch.cuda.mem_get_info()[0]
    if free < 24e9:
        pytest.skip("needs 24 GB")
    g = torch.Generator(device=DEV).manual_seed(5)
    k, v = (torch.randn(1, n, d, generator=g, device=DEV).to(torch.bfloat16) for _ in "kv")
    cu = np.array([0, rows - 300, rows], np.int64)
    blocks = rc.quantized_blocks(rows, 2)
    k8, v8 = (torch.full((1, rows, d), 0x7F, dtype=torch.uint8, device=DEV) for _ in "kv")
    ke, ve = (torch.full((1, blocks), 127, dtype=torch.uint8, device=DEV) for _ in "kv")
    lens = np.array([1, n])
    k2, v2 = (torch.cat([x[:, :1], x], 1) for x in (k, v))
    rc.quantize_kv(k2, v2, k8, v8, ke, ve, i32(cu), lens=i32(lens), cu_new=i32([0, 1, n + 1]))
    small_cu = prefix([1, n])
    k64, v64 = (pack(x, small_cu)[2] for x in (k2, v2))
    got = k8[0, rows - 300:rows - 300 + n].cpu().numpy()
    assert (np.abs(ref.VALUES[got]) <= 448).all()
    for q in (1, 3):
        w = AttendWorkload(seed=3, n_layers=1, n_q_heads=4, n_kv_heads=1, head_dim=d, dtype="bf16",
                           lengths=np.array([5], np.int32), req_res_off=np.array([0, 0, 0], np.int32),
                           req_res=np.zeros(0, np.int32), q_lens=np.array([1, q], np.int32),
                           ctx_lens=np.array([1, n], np.int32), mask=np.ones((1, 1, 1), np.uint8))
        qq = torch.randn(1 + q, 4, d, generator=g, device=DEV).to(torch.bfloat16)
        out, lse = torch.empty_like(qq), torch.empty(4, 1 + q, device=DEV)
        nb = rc.attend_workspace_bytes(2, q, n, n, 4, 1, d)
        ws = torch.empty(max(nb, 4) // 4, device=DEV)
        z = i32([0, 0, 0])
        one = torch.zeros(1, 5, d, dtype=torch.uint8, device=DEV)
        oe = torch.ones(1, 1, dtype=torch.uint8, device=DEV)
        rc.attend_quantized(qq, k8, v8, ke, ve, i32(w.cu_q), i32(cu), q, n, one, one, oe, oe, i32([0, 5]), z, i32([0]),
                            i32([0, 0]), 0, 1, out, ctx_len=i32(lens), max_route_len=1, lse=lse, workspace=ws, max_kv=n)
        want = ref.attend(w, qq.cpu().double().numpy(), np.zeros((1, 5, d)), np.zeros((1, 5, d)), k64, v64, 0,
                          ctx_off=small_cu)
        check_attend(out, lse, want, "past 4 GiB")
    del k8, v8
    torch.cuda.empty_cache()


# -------------------------------------------------------- streams and graphs

def test_a_step_on_another_stream_and_in_a_graph():
    """Append the newest token and attend, captured once and replayed on
    contexts that grow in place; every replay against the eager result."""
    w = small_attend(41, 3, 5, 8, 2, 128, "bf16", [1, 1, 1], [60, 1, 130], max_len=200)
    p, e = Packed(w, 0, slack=20), Packed(w, 0, slack=20)
    g = torch.Generator(device=DEV).manual_seed(9)
    ws, ws2 = p.workspace(), e.workspace()
    new = [torch.empty(3, 2, 128, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    cu_new = i32([0, 1, 2, 3])
    cu = i32(p.ctx_off)
    out = torch.zeros_like(p.q)

    def step(x, s, o, wk):
        x.ctx_len += 1
        rc.quantize_kv(new[0].transpose(0, 1), new[1].transpose(0, 1), x.ck, x.cv, x.cke, x.cve, cu, lens=x.ctx_len,
                       cu_new=cu_new, stream=s)
        w_, rt = x.w, x.rt
        rc.attend_quantized(x.q, x.ck, x.cv, x.cke, x.cve, rt.cu_q, cu, 1, 200, x.rk, x.rv, x.rke, x.rve, rt.cu_rows,
                            rt.route_off, rt.route_res, rt.route_tokens, 0, w_.n_layers, o, ctx_len=x.ctx_len,
                            max_route_len=max(rt.max_route_len, 1), workspace=wk, max_kv=x.mkv, stream=s)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    for t in new:
        t.normal_(generator=g)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(p, None, out, ws)
    torch.cuda.synchronize()
    for i in range(5):
        for t in new:
            t.copy_(torch.randn(t.shape, generator=g, device=DEV) * (1 + 3 * (i == 2)))
        p.q.copy_(torch.randn(p.q.shape, generator=g, device=DEV))
        e.q.copy_(p.q)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = torch.zeros_like(e.q)
        with torch.cuda.stream(side):
            step(e, side, want, ws2)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
        assert torch.equal(p.ck.view(torch.uint8), e.ck.view(torch.uint8)) and torch.equal(p.cke, e.cke)
        e.ck64, e.cv64 = (ref.dequantize(bits(c), bits(x), e.ctx_off, e.ctx_len.cpu().numpy())
                          for c, x in ((e.ck, e.cke), (e.cv, e.cve)))
        w.ctx_lens = e.ctx_len.cpu().numpy()
        check_attend(want, None, e.want(), i)
