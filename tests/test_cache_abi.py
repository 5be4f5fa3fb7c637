"""Checks that need no GPU: the plain definitions that the GPU tests use against
torch and closed forms, and the refusals of the cache-shrinking entry points
(every call below fails validation on the host, so that its made-up pointers
are never read)."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from paper_2608_19662_amd import recache as rc

FAKE = 0x1000


# ------------------------------------------------------------- the definitions

def test_round_e4m3_is_torchs():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(size=4000) * 2.0 ** rng.integers(-12, 6, 4000),
                        ref.VALUES[np.isfinite(ref.VALUES)], [2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -10, 0.0]])
    x = x.astype(np.float32).astype(np.float64)
    x = np.concatenate([x, (ref._POS[:-1] + ref._POS[1:]) / 2])  # every tie
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn)
    got = torch.from_numpy(ref.round_e4m3(x)).view(torch.float8_e4m3fn)
    assert torch.equal(want.float(), got.float())
    assert ref.round_e4m3(np.array([np.nan]))[0] == 127


@pytest.mark.parametrize("amax,e", [(0.0, 1), (448 * 2.0 ** -126, 1), (448.0, 127), (448.5, 128), (1.0, 119),
                                    (1.75, 119), (1.7501, 120), (2.0 ** -140, 1), (3.0e38, 247)])
def test_exponent(amax, e):
    assert ref.exponent(amax) == e


def test_quantize_error_is_half_a_step():
    """|value - x| is at most half a step of e4m3: 2^-4 |x| for normal codes, 2^-10 scales below."""
    rng = np.random.default_rng(2)
    x = rng.normal(size=(2, 200, 64)) * np.exp(rng.normal(size=(2, 200, 1)) * 3)
    cu = [0, 70, 200]
    codes, exps = np.zeros(x.shape, np.uint8), np.zeros((2, 200 // 64 + 2), np.uint8)
    ref.quantize(x, codes, exps, cu)
    y = ref.dequantize(codes, exps, cu)
    e = np.zeros((2, 200))
    for s in range(2):
        j = np.arange(cu[s + 1] - cu[s])
        e[:, cu[s]:cu[s + 1]] = exps[:, cu[s] // 64 + s + j // 64]
    assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * 2.0 ** (e - 127)[..., None])).all()


@pytest.mark.parametrize("seed", range(4))
def test_slots_are_never_shared(seed):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, 200, 50)
    cu = np.concatenate([[0], np.cumsum(lens)])
    seen = [int(cu[s]) // 64 + s + j for s in range(50) for j in range(-(-int(lens[s]) // 64))]
    assert len(set(seen)) == len(seen)
    assert max(seen) < rc.quantized_blocks(int(cu[-1]), 50)


def test_weights_of_a_row_sum_to_its_queries():
    """Every query gives 1 away: the weights sum to queries x heads."""
    from test_gpu_parity import small_attend

    w = small_attend(5, 3, 4, 4, 2, 64, "f32", [3, 1, 7], [9, 1, 30])
    q, ck, cv, rk, rv = (ref.host64(t) for t in w.layer_tensors(1))
    _, lse, _ = ref.attend(w, q, rk, rv, ck, cv, 1)
    rw, cw = ref.attend_weights(w, q, lse, rk, ck, 1)
    assert abs(rw.sum() + cw.sum() - 11 * 4) < 1e-9


def test_select_closed_forms():
    w = np.array([[1, 5, 5, 0, 2, np.nan, -1]], np.float32)
    assert list(ref.select(w, [0, 7], [0, 2], 0, 0)[0]) == [1, 2]
    assert list(ref.select(w, [0, 7], [0, 2], 0, 1)[0]) == [1, 6]
    assert list(ref.select(w, [0, 7], [0, 3], 1, 1)[0]) == [0, 1, 6]
    assert list(ref.select(w, [0, 7], [0, 6], 0, 0)[0]) == [0, 1, 2, 3, 4, 6]
    assert list(ref.select(w, [0, 3, 7], [0, 1, 1], 9, 9)[0]) == [2]


# ---------------------------------------------------------------- the refusals

def call(name, defaults, kw):
    a = dict(defaults)
    assert set(kw) <= set(a), set(kw) - set(a)
    a.update(kw)
    return getattr(rc.lib(), name)(*a.values())


USERS = dict(n_req=2, off=FAKE, res=FAKE, total=3, n_res=4, uo=FAKE, ur=FAKE, stream=None)
WEIGHTS = dict(dtype=1, layer=0, n_layers=2, n_req=2, cu_q=FAKE, cu_ctx=FAKE, total_q=4, max_q=3, Hq=32, Hkv=8,
               d=128, scale=0.0, q=FAKE, lse=FAKE, ck=FAKE, ctx_rows=10, cp=None, cw=FAKE, rk=FAKE, res_rows=10,
               rp=None, rw=FAKE, n_res=2, cu_kept=FAKE, res_off=None, mask=FAKE, uo=FAKE, ur=FAKE, n_users=3,
               stream=None)
SELECT = dict(n_seg=2, cu=FAKE, total=10, max_len=6, planes=8, w=FAKE, cu_kept=FAKE, total_kept=4, first=0, last=1,
              idx=FAKE, kw=None, ws=None, nb=0, stream=None)
QUANT = dict(dtype=1, n_seg=2, cu=FAKE, len=None, rows=10, planes=8, d=128, cu_new=None, src=10, k=FAKE, v=FAKE,
             rs=128, ps=1280, k8=FAKE, v8=FAKE, ke=FAKE, ve=FAKE, stream=None)
ATTEND = dict(dtype=1, layer=0, n_layers=1, n_req=2, cu_q=FAKE, cu_ctx=FAKE, ctx_len=None, total_q=4, max_q=3,
              max_ctx=9, max_kv=0, max_route_len=4, Hq=32, Hkv=8, d=128, scale=0.0, q=FAKE, ck=FAKE, cv=FAKE,
              cke=FAKE, cve=FAKE, ctx_rows=18, rk=FAKE, rv=FAKE, rke=FAKE, rve=FAKE, res_rows=10, n_res=2,
              cu_kept=FAKE, res_off=None, ro=FAKE, rr=FAKE, rt=FAKE, plan=None, out=FAKE, lse=None, ws=None, nb=0,
              stream=None)


@pytest.mark.parametrize("name,defaults,kw,code", [
    ("recache_resource_users", USERS, dict(n_req=0), rc.EINVAL),
    ("recache_resource_users", USERS, dict(n_res=0), rc.EINVAL),
    ("recache_resource_users", USERS, dict(total=-1), rc.EINVAL),
    ("recache_resource_users", USERS, dict(res=None), rc.EINVAL),
    ("recache_resource_users", USERS, dict(uo=None), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(dtype=2), rc.EUNSUPPORTED),
    ("recache_attend_weights", WEIGHTS, dict(d=96), rc.EUNSUPPORTED),
    ("recache_attend_weights", WEIGHTS, dict(Hq=30), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(Hq=72), rc.EUNSUPPORTED),
    ("recache_attend_weights", WEIGHTS, dict(layer=2), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(total_q=1), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(total_q=7), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(max_q=0), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(scale=float("inf")), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(cw=None, rw=None), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(ck=None), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(ctx_rows=0), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(rk=None), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(res_rows=0), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(mask=None), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(uo=None), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(ur=None), rc.EINVAL),
    ("recache_attend_weights", WEIGHTS, dict(lse=None), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(n_seg=0), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(planes=0), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(total_kept=11), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(max_len=11), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(first=-1), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(last=-1), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(w=None), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(idx=None), rc.EINVAL),
    ("recache_select_kept", SELECT, dict(total=300000, max_len=200000), rc.EWORKSPACE),
    ("recache_select_kept", SELECT, dict(total=300000, max_len=200000, ws=FAKE, nb=100), rc.EWORKSPACE),
    ("recache_select_kept", SELECT, dict(total=300000, max_len=200000, ws=FAKE + 4, nb=1 << 30), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(dtype=2), rc.EUNSUPPORTED),
    ("recache_quantize_kv", QUANT, dict(d=32), rc.EUNSUPPORTED),
    ("recache_quantize_kv", QUANT, dict(n_seg=0), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(planes=0), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(rows=-1), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(cu=None), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(k=None), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(ve=None), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(rs=127), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(ps=-128), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(rs=1 << 22), rc.EUNSUPPORTED),
    ("recache_quantize_kv", QUANT, dict(k=FAKE + 8), rc.EINVAL),
    ("recache_quantize_kv", QUANT, dict(v8=FAKE + 4), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(dtype=0), rc.EUNSUPPORTED),
    ("recache_attend_quantized", ATTEND, dict(d=256), rc.EUNSUPPORTED),
    ("recache_attend_quantized", ATTEND, dict(Hq=72), rc.EUNSUPPORTED),
    ("recache_attend_quantized", ATTEND, dict(max_q=10), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(total_q=1), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(max_route_len=1025), rc.EUNSUPPORTED),
    ("recache_attend_quantized", ATTEND, dict(ctx_rows=0), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(res_rows=0), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(cke=None), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(rve=None), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(res_rows=0, res_off=FAKE, rke=None), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(n_res=-1), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(n_res=0), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(plan=FAKE + 2), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(out=None), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(ck=FAKE + 8), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(scale=float("nan")), rc.EINVAL),
    ("recache_attend_quantized", ATTEND, dict(max_q=1, total_q=2), rc.EWORKSPACE),
    ("recache_attend_quantized", ATTEND, dict(max_q=1, total_q=2, ws=FAKE, nb=64), rc.EWORKSPACE),
])
def test_refusals(name, defaults, kw, code):
    assert call(name, defaults, kw) == code
    assert rc.last_error()


def test_nothing_to_do_is_fine():
    assert call("recache_select_kept", SELECT, dict(total=0, max_len=0, total_kept=0, w=None, idx=None)) == rc.OK
    assert call("recache_quantize_kv", QUANT, dict(rows=0, src=0, k=None, v=None)) == rc.OK
    assert rc.last_error() == ""


def test_sizes():
    assert rc.quantized_blocks(0, 3) == 3
    assert rc.quantized_blocks(63, 1) == 1
    assert rc.quantized_blocks(64, 1) == 2
    assert rc.quantized_blocks(2 ** 31 - 1, 16384) == (2 ** 31 - 1) // 64 + 16384
    assert rc.select_workspace_bytes(4, 100000, 300) == 0
    assert rc.select_workspace_bytes(4, 100000, 99000) >= 400000


def test_binding_refuses_host_tensors_and_wrong_shapes():
    z = lambda *s, **k: torch.zeros(*s, **k)
    i = lambda n: z(n, dtype=torch.int32)
    with pytest.raises(TypeError):
        rc.quantize_kv(z(2, 8, 64), z(2, 8, 64), z(2, 8, 64, dtype=torch.uint8), z(2, 8, 64, dtype=torch.uint8),
                       z(2, 1, dtype=torch.uint8), z(2, 1, dtype=torch.uint8), i(2))
    with pytest.raises(ValueError):  # scale bytes of another shape
        rc.quantize_kv(z(2, 8, 64), z(2, 8, 64), z(2, 8, 64, dtype=torch.uint8), z(2, 8, 64, dtype=torch.uint8),
                       z(2, 2, dtype=torch.uint8), z(2, 2, dtype=torch.uint8), i(2))
    with pytest.raises(ValueError):  # more source rows than the cache, no offsets for them
        rc.quantize_kv(z(2, 9, 64), z(2, 9, 64), z(2, 8, 64, dtype=torch.uint8), z(2, 8, 64, dtype=torch.uint8),
                       z(2, 1, dtype=torch.uint8), z(2, 1, dtype=torch.uint8), i(2))
    with pytest.raises(TypeError):
        rc.select_kept(z(8, 10), i(2), i(2), i(3), max_len=10)
    with pytest.raises(ValueError):
        rc.select_kept(z(8, 10), i(2), i(3), i(3), max_len=10)
    with pytest.raises(ValueError):
        rc.attend_weights(z(4, 4, 64), z(4, 4), i(2), i(2), 4, None, None, None, None, 0, ctx_k=z(2, 4, 64))
    with pytest.raises(TypeError):
        rc.resource_users(i(2), i(3), 4, i(5), i(3))
