"""Host side of the eight-bit operators and the norm: sizes and refusals, without a GPU."""
import ctypes

import pytest

from paper_2505_11204_b200 import build, randes


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def refused(code, f):
    with pytest.raises(randes.RandesError) as e:
        f()
    assert e.value.code == code, e.value


def test_sizes():
    size = randes.randes_packed_eight_bytes
    assert size(1, 1) == 128 * 128 + 512
    assert size(128, 512) == 4 * 16384 + 512 and size(129, 512) == 2 * size(128, 512)
    assert size(128, 513) == 5 * 16384 + 2 * 512
    assert size(0, 5) == size(5, 0) == 0
    assert size(1 << 31, 1 << 31) == 0 and size(0xFFFFFFFF, 1) == 0 and size(1 << 20, 1 << 18) == (1 << 38) + (1 << 38) // 128
    assert randes.randes_packed_eight_linear_workspace(700, randes.EIGHT_BITS, 10000) == 0
    assert randes.randes_packed_eight_linear_workspace(700, randes.BF16, 16) == 0
    assert randes.randes_packed_eight_linear_workspace(700, randes.F32, 17) == size(17, 700)
    assert randes.randes_rms_norm_backward_workspace(1, 1) == randes.randes_rms_norm_backward_workspace(256, 1024) == 0
    for rows, cols in ((257, 1024), (1000, 768), (10 ** 6, 4096), (3, 32768)):
        assert randes.randes_rms_norm_backward_workspace(rows, cols) >= 4 * cols


def test_structures_have_the_header_sizes():
    assert ctypes.sizeof(randes.RmsNorm) == 120 and len(randes._NORM(*[0] * 16, 1e-6)) == 120
    assert ctypes.sizeof(randes.RmsNormBackward) == 112 and len(randes._NORM_BACKWARD(*[0] * 16)) == 112
    assert len(randes._ONE_MATRIX(0, 0, 0, 0)) == ctypes.sizeof(randes.Matrix) and len(randes._ONE_ADDRESS(0)) == ctypes.sizeof(ctypes.c_void_p)


def test_pack_and_transpose_refusals():
    inv, mis = randes.INVALID_ARGUMENT, randes.MISALIGNED
    m = lambda data=4096, rows=4, cols=300, stride=300: (randes.Matrix * 1)((data, rows, cols, stride))
    p = lambda a=1 << 20: (ctypes.c_void_p * 1)(a)
    pack = lambda mats=m(), n=1, dt=0, to=p(): randes.randes_pack_eight(mats, n, dt, to, None)
    refused(inv, lambda: pack(mats=None))
    refused(inv, lambda: pack(to=None))
    refused(inv, lambda: pack(mats=m(data=None)))
    refused(inv, lambda: pack(to=p(None)))
    refused(inv, lambda: pack(mats=m(stride=299)))
    refused(inv, lambda: pack(mats=m(rows=1 << 31, cols=1 << 31, stride=1 << 31)))
    refused(inv, lambda: pack(to=p(4096 + 16)))
    refused(mis, lambda: pack(to=p((1 << 20) + 8)))
    refused(mis, lambda: pack(mats=m(data=4098)))
    refused(randes.UNSUPPORTED_DTYPE, lambda: pack(dt=2))
    pack(n=0, mats=None, to=None)
    pack(mats=m(rows=0, data=None), to=p(None))
    unpack = lambda mats=m(), dt=0, frm=p(): randes.randes_unpack_eight(frm, 1, mats, dt, None)
    refused(inv, lambda: unpack(frm=p(None)))
    refused(mis, lambda: unpack(frm=p((1 << 20) + 4)))
    refused(randes.UNSUPPORTED_DTYPE, lambda: unpack(dt=7))
    turn = lambda mat=m(), dt=0, a=None, t=1 << 20: randes.randes_pack_eight_transposed(mat, dt, a, t, None)
    refused(inv, lambda: turn(mat=None))
    refused(inv, lambda: turn(t=None))
    refused(inv, lambda: turn(a=1 << 20))
    refused(inv, lambda: turn(t=4096))
    refused(mis, lambda: turn(a=1 << 21, t=(1 << 20) + 2))
    refused(inv, lambda: randes.randes_transpose_eight(1 << 20, 4, 300, 1 << 20, None))
    refused(mis, lambda: randes.randes_transpose_eight((1 << 20) + 8, 4, 300, 1 << 22, None))
    randes.randes_transpose_eight(None, 0, 300, None, None)


def test_retrieval_refusals():
    plan = randes.Plan([4, 4], [300, 300], [0, 0], [3], task_ids=[7], seeds=[1], host_only=True)
    base, layers = (ctypes.c_void_p * 2)(1 << 12, 1 << 14), (ctypes.c_uint32 * 1)(1)
    call = lambda task=7, ls=layers, b=base, M=1 << 20, to=(ctypes.c_void_p * 1)(1 << 22): randes.randes_retrieve_packed_eight(plan.handle, task, 0.5, ls, 1, b, M, to, None)
    refused(randes.UNKNOWN_TASK, lambda: call(task=8))
    refused(randes.INVALID_ARGUMENT, lambda: call(ls=(ctypes.c_uint32 * 1)(2)))
    refused(randes.INVALID_ARGUMENT, lambda: call(ls=None))
    refused(randes.INVALID_ARGUMENT, lambda: call(b=None))
    refused(randes.INVALID_ARGUMENT, lambda: call(M=None))
    refused(randes.INVALID_ARGUMENT, lambda: call(to=(ctypes.c_void_p * 1)(1 << 20)))
    refused(randes.MISALIGNED, lambda: call(to=(ctypes.c_void_p * 1)((1 << 22) + 8)))
    gauss = randes.Plan([4], [300], [0], [randes.GAUSS], task_ids=[7], seeds=[1], host_only=True)
    refused(randes.INVALID_ARGUMENT, lambda: randes.randes_retrieve_packed_eight(gauss.handle, 7, 0.5, (ctypes.c_uint32 * 1)(0), 1, base, 1 << 20, (ctypes.c_void_p * 1)(1 << 22), None))


def test_norm_refusals():
    inv, mis = randes.INVALID_ARGUMENT, randes.MISALIGNED
    ok = dict(x=1 << 12, y=1 << 20, x_stride=256, y_stride=256, rows=4, cols=256, eps=1e-6)
    norm = lambda **kw: randes.randes_rms_norm(randes.RmsNorm(**{**ok, **kw}), None)
    for kw, code in ((dict(cols=0), inv), (dict(cols=32769, x_stride=32769, y_stride=32769), inv), (dict(eps=0.0), inv), (dict(eps=2.0), inv), (dict(eps=float("nan")), inv),
                     (dict(x=None), inv), (dict(x_stride=255), inv), (dict(y=1 << 12, y_stride=300), inv), (dict(y=(1 << 12) + 64), inv), (dict(h=1 << 20, h_stride=256), inv),
                     (dict(y8=(1 << 21) + 8), mis), (dict(y8=1 << 20), inv), (dict(kept8=1 << 22, y8=(1 << 22) + 16), inv), (dict(rstd=2), mis), (dict(gain=6, gain_dtype=0), mis),
                     (dict(dtype=3), randes.UNSUPPORTED_DTYPE), (dict(gain=16, gain_dtype=3), randes.UNSUPPORTED_DTYPE), (dict(residual=1 << 13, residual_stride=10), inv)):
        refused(code, lambda: norm(**kw))
    norm(rows=0, x=None, y=None)
    refused(inv, lambda: randes._check(randes.lib().randes_rms_norm(None, None)))
    ok2 = dict(dy=1 << 12, h=1 << 14, rstd=1 << 16, dx=1 << 18, dy_stride=256, h_stride=256, dx_stride=256, rows=4, cols=256)
    many = dict(rows=2000, dy=1 << 30, h=1 << 31, dx=1 << 32)
    back = lambda at=None, n=0, **kw: randes.randes_rms_norm_backward(randes.RmsNormBackward(**{**ok2, **kw}), at, n, None)
    for kw, code in ((dict(h=None), inv), (dict(kept8=1 << 20), inv), (dict(h=None, kept8=(1 << 20) + 4), mis), (dict(rstd=None), inv), (dict(rstd=5), mis), (dict(dx=None), inv),
                     (dict(dy=None), inv), (dict(dx=(1 << 12) + 64), inv), (dict(h=None, kept8=1 << 18), inv), (dict(many, dgain=1 << 34), randes.WORKSPACE_TOO_SMALL),
                     (dict(many, dgain=1 << 34, at=(1 << 35) + 8, n=1 << 24), mis), (dict(dgain=3), mis), (dict(dtype=9), randes.UNSUPPORTED_DTYPE)):
        refused(code, lambda: back(**kw))
    back(rows=0, dx=None, h=None)


def test_product_refusals():
    inv, mis = randes.INVALID_ARGUMENT, randes.MISALIGNED
    ok = dict(w=1 << 20, rows=8, cols=256, x=1 << 22, n_tokens=4, y=1 << 24, y_dtype=0, y_stride=8, stream=None)
    call = lambda **kw: randes.randes_packed_eight_linear(**{**ok, **kw})
    for kw, code in ((dict(w=None), inv), (dict(x=None), inv), (dict(y=None), inv), (dict(w=(1 << 20) + 8), mis), (dict(x=(1 << 22) + 8), mis), (dict(y=(1 << 24) + 1), mis),
                     (dict(y_stride=7), inv), (dict(y_dtype=8), randes.UNSUPPORTED_DTYPE), (dict(x_dtype=2), randes.UNSUPPORTED_DTYPE), (dict(y=1 << 20), inv), (dict(y=1 << 22), inv),
                     (dict(x_dtype=0, x_stride=255), inv), (dict(n_tokens=17, x_dtype=1, x_stride=256), randes.WORKSPACE_TOO_SMALL), (dict(rows=1 << 31, cols=1 << 31), inv),
                     (dict(n_tokens=17, x_dtype=1, x_stride=256, workspace=(1 << 26) + 8, workspace_bytes=1 << 20), mis),
                     (dict(n_tokens=17, x_dtype=1, x_stride=256, workspace=1 << 24, workspace_bytes=1 << 20), inv)):
        refused(code, lambda: call(**kw))
    call(n_tokens=0, x=None, y=None)
    call(rows=0, w=None, y=None)


def test_the_first_call_of_a_process_may_be_any(monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(randes, "_torch", None)      # as a process that has made no call on tensors finds it
    p = randes._new_packed8(3, 200, torch.device("cpu"))
    assert (p.rows, p.cols, p.nbytes) == (3, 200, randes.randes_packed_eight_bytes(3, 200)) and p.data.dtype is torch.uint8
