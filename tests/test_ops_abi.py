"""acp_ops.h on the CPU: exported symbols, layouts, host tables, and the refusal of bad
arguments before anything is launched."""
import ctypes
import math

import pytest
import torch

from paper_2504_06949_amd import acp, ops
from tests._helpers import ensure_built

BIG = 1 << 46


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()
    ops.lib()


def test_every_declared_symbol_is_exported():
    assert set(ops.header_functions()) == set(ops._SIGS)
    lib = ctypes.CDLL(acp.LIB_PATH)
    for n in ops.header_functions():
        assert hasattr(lib, n), n


def _norm_fwd(**kw):
    a = dict(x=16, xs=None, w=16, b=None, dt=1, wdt=0, B=1, H=2, L=3, n=64, per=1, center=1, eps=1e-5, y=32,
             mean=16, rstd=16, stream=None)
    a.update(kw)
    return ops.lib().acp_norm_fwd(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(x=0), acp.ACP_EINVAL), (dict(x=17), acp.ACP_EINVAL), (dict(w=0), acp.ACP_EINVAL),
    (dict(y=0), acp.ACP_EINVAL), (dict(y=16), acp.ACP_EINVAL), (dict(dt=5), acp.ACP_EINVAL),
    (dict(wdt=2), acp.ACP_EINVAL), (dict(B=-1), acp.ACP_EINVAL), (dict(n=0), acp.ACP_EINVAL),
    (dict(eps=-1.0), acp.ACP_EINVAL), (dict(eps=math.nan), acp.ACP_EINVAL),
    (dict(eps=math.inf), acp.ACP_EINVAL), (dict(rstd=None), acp.ACP_EINVAL),
    (dict(mean=None), acp.ACP_EINVAL), (dict(center=0), acp.ACP_EINVAL),
    (dict(xs=(ctypes.c_int64 * 3)(64, -1, 64)), acp.ACP_EINVAL),
    (dict(n=16385), acp.ACP_EUNSUPPORTED), (dict(H=65536), acp.ACP_EUNSUPPORTED),
    (dict(B=65536, L=65536, H=1), acp.ACP_EUNSUPPORTED),
    (dict(L=0, x=0, y=0), acp.ACP_OK),
])
def test_norm_forward_refusals(kw, status):
    assert _norm_fwd(**kw) == status
    assert (acp.acp_last_error() == "") == (status == acp.ACP_OK)


def _norm_bwd(**kw):
    a = dict(dy=16, dys=None, x=32, xs=None, w=16, dt=1, wdt=0, B=1, H=2, L=3, n=64, per=1, mean=16, rstd=16,
             dx=48, dxs=None, dw=16, db=16, ws=16, ws_bytes=BIG, stream=None)
    a.update(kw)
    return ops.lib().acp_norm_bwd(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(dy=0), acp.ACP_EINVAL), (dict(x=0), acp.ACP_EINVAL), (dict(rstd=0), acp.ACP_EINVAL),
    (dict(dx=0), acp.ACP_EINVAL), (dict(dx=32), acp.ACP_EINVAL), (dict(dw=0), acp.ACP_EINVAL),
    (dict(db=2), acp.ACP_EINVAL), (dict(ws=0), acp.ACP_EINVAL),
    (dict(dx=16, dxs=(ctypes.c_int64 * 3)(0, 64, 128)), acp.ACP_EINVAL),   # dy's place, other strides
    (dict(ws_bytes=8), acp.ACP_EWORKSPACE), (dict(n=20000), acp.ACP_EUNSUPPORTED),
])
def test_norm_backward_refusals(kw, status):
    assert _norm_bwd(**kw) == status
    assert acp.acp_last_error() != ""


@pytest.mark.parametrize("args", [
    (3, 1e4, 0, 1.0, 0.0, 1.0, 32.0), (0, 1e4, 0, 1.0, 0.0, 1.0, 32.0), (64, 1.0, 0, 1.0, 0.0, 1.0, 32.0),
    (64, math.inf, 0, 1.0, 0.0, 1.0, 32.0), (64, 1e4, 4, 1.0, 0.0, 1.0, 32.0),
    (64, 1e4, 1, 0.5, 0.0, 1.0, 32.0), (2, 1e4, 2, 2.0, 0.0, 1.0, 32.0), (64, 1e4, 3, 2.0, 0.0, 1.0, 32.0),
    (64, 1e4, 3, 2.0, 4096.0, 32.0, 32.0),
])
def test_rotary_table_refusals(args):
    out = (ctypes.c_double * 64)()
    assert ops.lib().acp_rotary_table(*args, out) == acp.ACP_EINVAL
    assert acp.acp_last_error() != ""


def test_rotary_tables():
    """Against the formulas; the ends of the ramp are exactly the unscaled and the linear table."""
    def table(scaling, factor=1.0, train_len=0.0, slow=1.0, fast=32.0, rot=64):
        out = (ctypes.c_double * (rot // 2))()
        acp._check(ops.lib().acp_rotary_table(rot, 1e4, scaling, factor, train_len, slow, fast, out))
        return list(out)

    plain = table(0)
    for i, t in enumerate(plain):
        assert math.isclose(t, 10000.0 ** (-i / 32) / (2 * math.pi), rel_tol=1e-14)
    assert table(1, 4.0) == [t / 4.0 for t in plain]
    scaled = table(2, 8.0)
    assert scaled[0] == plain[0] and math.isclose(scaled[-1], plain[-1] / 8.0, rel_tol=1e-13)
    ramp = table(3, 8.0, 4096.0)
    for t, p in zip(ramp, plain):
        r = 4096.0 * p
        want = p if r >= 32.0 else p / 8.0 if r <= 1.0 else p * ((r - 1) / 31) + p / 8 * (1 - (r - 1) / 31)
        assert math.isclose(t, want, rel_tol=1e-14)
    assert ramp[0] == plain[0] and ramp[-1] == plain[-1] / 8.0


def _rotary(**kw):
    a = dict(q=16, qs=None, k=32, ks=None, dt=1, B=1, H=2, Hk=2, L=3, d=64, rot=64, layout=0, inverse=0,
             amp=1.0, turns=16, pos=16, pos_bytes=4, ps=(ctypes.c_int64 * 2)(0, 1), start=0, qo=48, qos=None,
             ko=64, kos=None, stream=None)
    a.update(kw)
    return ops.lib().acp_rotary(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(q=0, k=0), acp.ACP_EINVAL), (dict(qo=0), acp.ACP_EINVAL), (dict(ko=65), acp.ACP_EINVAL),
    (dict(dt=3), acp.ACP_EINVAL), (dict(rot=66), acp.ACP_EINVAL), (dict(rot=3), acp.ACP_EINVAL),
    (dict(rot=0), acp.ACP_EINVAL), (dict(layout=2), acp.ACP_EINVAL), (dict(amp=math.nan), acp.ACP_EINVAL),
    (dict(turns=0), acp.ACP_EINVAL), (dict(pos_bytes=2), acp.ACP_EINVAL), (dict(ps=None), acp.ACP_EINVAL),
    (dict(ps=(ctypes.c_int64 * 2)(0, -1)), acp.ACP_EINVAL), (dict(pos=None, start=1 << 31), acp.ACP_EINVAL),
    (dict(qo=16, qos=(ctypes.c_int64 * 3)(0, 64, 128)), acp.ACP_EINVAL),
    (dict(d=63, rot=2), acp.ACP_EUNSUPPORTED), (dict(d=2048), acp.ACP_EUNSUPPORTED),
    (dict(H=65535), acp.ACP_EUNSUPPORTED), (dict(L=0), acp.ACP_OK),
])
def test_rotary_refusals(kw, status):
    assert _rotary(**kw) == status


def test_paged_layout():
    n = ctypes.c_size_t(0)
    y = ops.PagedLayout()
    acp._check(ops.lib().acp_paged_cache_size(5, 6, 3, 64, acp.ACP_BF16, ctypes.byref(n)))
    acp._check(ops.lib().acp_paged_offsets(5, 6, 3, 64, acp.ACP_BF16, ctypes.byref(y)))
    kv = 5 * 3 * 64 * 64 * 2
    assert (y.k, y.v, y.c, y.total) == (0, kv, 2 * kv, 2 * kv + 5 * 6 * 64 * 8) and n.value == y.total
    for args, status in (((0, 6, 3, 64, 1), acp.ACP_EINVAL), ((5, 6, 4, 64, 1), acp.ACP_EUNSUPPORTED),
                         ((5, 34, 2, 64, 1), acp.ACP_EUNSUPPORTED), ((5, 6, 3, 96, 1), acp.ACP_EUNSUPPORTED),
                         ((5, 6, 3, 64, 9), acp.ACP_EINVAL)):
        assert ops.lib().acp_paged_cache_size(*args, ctypes.byref(n)) == status


def _append(**kw):
    a = dict(k=16, ks=None, v=16, vs=None, f=16, fs=None, dt=1, T=4, N=2, W=3, P=9, H=4, Hk=2, d=64, cu=16,
             past=16, table=16, cache=16, cache_bytes=BIG, flags=None, stream=None)
    a.update(kw)
    return ops.lib().acp_paged_append(*a.values())


def _attend(**kw):
    a = dict(q=16, qs=None, dt=1, T=4, N=2, W=3, P=9, H=4, Hk=2, d=64, cu=16, past=16, table=16, cache=16,
             cache_bytes=BIG, gq=16, gk=16, eps=1e-4, L_max=1000, max_new=2, max_len=4096, O=16, lse=16,
             flags=None, ws=16, ws_bytes=BIG, stream=None)
    a.update(kw)
    return ops.lib().fox_attn_paged(*a.values())


@pytest.mark.parametrize("kw,status", [
    (dict(k=0), acp.ACP_EINVAL), (dict(v=8), acp.ACP_EINVAL), (dict(f=0), acp.ACP_EINVAL),
    (dict(cu=0), acp.ACP_EINVAL), (dict(past=2), acp.ACP_EINVAL), (dict(table=0), acp.ACP_EINVAL),
    (dict(cache=0), acp.ACP_EINVAL), (dict(flags=1), acp.ACP_EINVAL), (dict(T=-1), acp.ACP_EINVAL),
    (dict(ks=(ctypes.c_int64 * 2)(100, 64)), acp.ACP_EINVAL),      # rows not 16-byte aligned
    (dict(vs=(ctypes.c_int64 * 2)(-128, 64)), acp.ACP_EINVAL),
    (dict(fs=(ctypes.c_int64 * 2)(1, -1)), acp.ACP_EINVAL),
    (dict(T=(1 << 26) + 1), acp.ACP_EUNSUPPORTED), (dict(N=65536), acp.ACP_EUNSUPPORTED),
    (dict(H=5), acp.ACP_EUNSUPPORTED), (dict(cache_bytes=100), acp.ACP_EWORKSPACE),
    (dict(N=0, past=0, table=0), acp.ACP_OK),
])
def test_append_refusals(kw, status):
    assert _append(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), acp.ACP_EINVAL), (dict(q=24), acp.ACP_EINVAL), (dict(O=0), acp.ACP_EINVAL),
    (dict(lse=0), acp.ACP_EINVAL), (dict(gq=0), acp.ACP_EINVAL), (dict(gk=None), acp.ACP_EINVAL),
    (dict(eps=1.0), acp.ACP_EINVAL), (dict(eps=math.nan), acp.ACP_EINVAL), (dict(L_max=0), acp.ACP_EINVAL),
    (dict(max_new=-1), acp.ACP_EINVAL), (dict(max_len=-1), acp.ACP_EINVAL),
    (dict(qs=(ctypes.c_int64 * 2)(4, 64)), acp.ACP_EINVAL), (dict(cache_bytes=0), acp.ACP_EWORKSPACE),
    (dict(max_len=100000, ws_bytes=16), acp.ACP_EWORKSPACE), (dict(d=80), acp.ACP_EUNSUPPORTED),
    (dict(T=1 << 25, H=16, Hk=16), acp.ACP_EUNSUPPORTED), (dict(N=0, past=0, table=0), acp.ACP_OK),
])
def test_attend_refusals(kw, status):
    assert _attend(**kw) == status


def test_tensor_helpers_refuse_cpu_tensors():
    x, w = torch.zeros(2, 3, 4, 64), torch.ones(64)
    for f in (lambda: ops.rms_norm(x, w), lambda: ops.layer_norm(x, w, w),
              lambda: ops.norm_backward(x, x, w, None, torch.zeros(2, 3, 4)),
              lambda: ops.Rotary(64, device="cpu").forward(x),
              lambda: ops.PagedCache(2, 3, 64, device="cpu").append(
                  x[0].bfloat16(), x[0].bfloat16(), torch.zeros(2, 3), torch.zeros(2).int(), torch.zeros(1).int(),
                  torch.zeros(1, 1).int())):
        with pytest.raises(ValueError, match="GPU"):
            f()
    with pytest.raises(acp.AcpError):
        ops.Rotary(7, device="cpu")
    with pytest.raises(acp.AcpError):
        ops.PagedCache(4, 4, 80, device="cpu")
    with pytest.raises(TypeError):
        ops.PagedCache(4, 4, 64, dtype=torch.float16, device="cpu")


@pytest.mark.parametrize("call,status", [
    (lambda: _norm_fwd(B=1 << 15, L=(1 << 15) + 1, H=1), acp.ACP_EUNSUPPORTED),
    (lambda: _norm_fwd(B=46340, L=46340, H=1, n=1), acp.ACP_EUNSUPPORTED),      # just under 2^31
    (lambda: _rotary(pos=None, start=(1 << 63) - 1), acp.ACP_EINVAL),
    (lambda: _rotary(pos=None, start=(1 << 31) - 2), acp.ACP_EINVAL),
    (lambda: _rotary(ko=48), acp.ACP_EINVAL),                                    # both into one place
    (lambda: _rotary(amp=1e300), acp.ACP_EINVAL),
    (lambda: _rotary(B=1 << 15, L=1 << 14, d=64), acp.ACP_EUNSUPPORTED),
    (lambda: _append(T=1 << 25, H=4), acp.ACP_EUNSUPPORTED),
    (lambda: _append(N=65535, H=128, Hk=128), acp.ACP_EUNSUPPORTED),
    (lambda: _attend(N=65535, H=128, Hk=128), acp.ACP_EUNSUPPORTED),
    (lambda: _attend(T=1 << 25), acp.ACP_EUNSUPPORTED),
    (lambda: _attend(max_len=(1 << 31) + 1), acp.ACP_EINVAL),
])
def test_bounds_of_sizes(call, status):
    """Counts that an int or a launch could not hold are refused."""
    assert call() == status and acp.acp_last_error() != ""


def test_workspace_sizes_of_empty_calls():
    n = ctypes.c_size_t(7)
    for B, H, L, per in ((0, 3, 5, 1), (2, 0, 5, 1), (2, 0, 5, 0), (2, 3, 0, 1)):
        assert ops.lib().acp_norm_workspace_size(B, H, L, 64, per, ctypes.byref(n)) == acp.ACP_OK
        assert n.value == 0
    for T, N in ((0, 0), (0, 3), (5, 0)):
        assert ops.lib().acp_paged_workspace_size(T, N, 4, 2, 64, 1, 0, 0, ctypes.byref(n)) == acp.ACP_OK


def test_operator_timing_without_launches():
    acp.acp_timing_reset()
    assert ops.acp_op_timing_read() == {n: (0, 0.0) for n in ops.OP_NAMES}


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), acp.ACP_EINVAL), (dict(O=8), acp.ACP_EINVAL), (dict(eps=1.0), acp.ACP_EINVAL),
    (dict(ws=0), acp.ACP_EINVAL), (dict(ws_bytes=16), acp.ACP_EWORKSPACE), (dict(d=80), acp.ACP_EUNSUPPORTED),
    (dict(T=0, N=0, past=0, table=0, q=0, O=0), acp.ACP_OK),
])
def test_attention_with_filled_rows_refuses_the_same(kw, status, monkeypatch):
    monkeypatch.setattr(ops.lib(), "fox_attn_paged", ops.lib().fox_attn_paged_filled)
    assert _attend(**kw) == status
