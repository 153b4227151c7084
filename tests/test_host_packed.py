"""Host-side checks of the four-bit weights and token scores that need no GPU: sizes, and arguments refused before anything
is launched (the addresses below are never read)."""
import ctypes

import pytest

from paper_2505_11204_b200 import build, randes

INV, MIS, DT, WS = randes.INVALID_ARGUMENT, randes.MISALIGNED, randes.UNSUPPORTED_DTYPE, randes.WORKSPACE_TOO_SMALL


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def _refused(code, fn):
    with pytest.raises(randes.RandesError) as e:
        fn()
    assert e.value.code == code, (e.value.code, str(e.value))
    assert randes.randes_last_error()


def test_packed_sizes():
    for rows, cols in ((64, 64), (1, 1), (65, 130), (50257, 768), (128, 128)):
        blocks = -(-rows // 64)
        assert randes.randes_packed_bytes(rows, cols, 32) == blocks * -(-cols // 64) * (2048 + 256)
        assert randes.randes_packed_bytes(rows, cols, 64) == blocks * -(-cols // 64) * (2048 + 128)
        assert randes.randes_packed_bytes(rows, cols, 128) == blocks * -(-cols // 128) * (4096 + 128)
    # half a byte and two bytes of scale per 64 columns
    assert abs(randes.randes_packed_bytes(8192, 8192, 64) / 8192 ** 2 - (0.5 + 2 / 64)) < 1e-9
    for bad in ((0, 64, 64), (64, 0, 64), (64, 64, 16), (64, 64, 0), (70000, 70000, 64)):
        assert randes.randes_packed_bytes(*bad) == 0


def test_workspace_sizes():
    f = randes.randes_packed_linear_workspace
    assert f(512, 4096, randes.F32, 0, True) == f(512, 4096, randes.F32, 8, True) == f(1 << 16, 1 << 15, randes.BF16, 8, True) == 0
    assert f(512, 4096, randes.BF16, 17, False) == 24 * 4096 * 2            # whole groups of eight rows
    assert f(512, 4100, randes.F32, 64, False) == 64 * 4160 * 2 * 3         # whole tiles of columns, three terms
    assert f(512, 4096, randes.BF16, 1000, False) == f(512, 4096, randes.BF16, 64, False)
    assert f(512, 4096, randes.BF16, 64, True) > f(512, 4096, randes.BF16, 64, False)
    # few fp32 tokens need one where the matrix (with a superposition: both matrices) is large
    assert f(1 << 13, 1 << 12, randes.F32, 1, False) == 8 * 4096 * 2 * 3
    assert f(1 << 13, (1 << 12) - 1, randes.F32, 1, False) == 0 < f(1 << 13, (1 << 12) - 1, randes.F32, 1, True)
    assert f(50257, 768, randes.F32, 1, False) == f(50257, 767, randes.F32, 1, True) == 0


def test_pack_arguments():
    arr = lambda *a: (ctypes.c_void_p * len(a))(*a)
    mat = lambda data=0x10000, rows=8, cols=64, stride=64: (randes.Matrix * 1)((data, rows, cols, stride))
    call = lambda m, n=1, dt=0, group=64, to=arr(0x100000): randes.randes_pack(m, n, dt, group, to, None)
    _refused(DT, lambda: call(mat(), dt=3))
    _refused(INV, lambda: call(mat(), group=65))
    _refused(INV, lambda: call(None))
    _refused(INV, lambda: call(mat(), to=None))
    _refused(INV, lambda: call(mat(data=None)))
    _refused(MIS, lambda: call(mat(data=0x10002)))
    _refused(INV, lambda: call(mat(stride=63)))
    _refused(INV, lambda: call(mat(stride=1 << 41)))
    _refused(INV, lambda: call(mat(rows=70000, cols=70000, stride=70000)))
    _refused(INV, lambda: call(mat(), to=arr(None)))
    _refused(MIS, lambda: call(mat(), to=arr(0x100008)))
    _refused(INV, lambda: call(mat(data=0x100000 + 2048)))                  # inside the packed buffer
    call(None, n=0)                                                         # nothing to do
    call(mat(data=None, rows=0))
    _refused(DT, lambda: randes.randes_unpack(arr(0x100000), 1, 64, mat(), 2, None))
    _refused(INV, lambda: randes.randes_unpack(arr(0x100000), 1, 7, mat(), 0, None))


def test_plan_level_arguments():
    plan = randes.Plan([32, 32], [128, 128], [0, 0], [randes.SHUFFLE | randes.FLIP], task_ids=[5], seeds=[1], host_only=True)
    base = (ctypes.c_void_p * 2)(0x10000, 0x20000)
    layers, to = (ctypes.c_uint32 * 1)(1), (ctypes.c_void_p * 1)(0x100000)
    call = lambda task=5, n=1, b=base, M=0x1000000, group=64, ls=layers, dst=to: \
        randes.randes_retrieve_packed(plan.handle, task, 1.0, ls, n, b, M, group, dst, None)
    _refused(randes.UNKNOWN_TASK, lambda: call(task=6))
    _refused(INV, lambda: call(ls=(ctypes.c_uint32 * 1)(2)))
    _refused(INV, lambda: call(group=1))
    _refused(INV, lambda: call(M=None))
    _refused(MIS, lambda: call(M=0x1000010))
    _refused(INV, lambda: call(b=None))
    _refused(INV, lambda: call(b=(ctypes.c_void_p * 2)(0x10000, None)))
    _refused(INV, lambda: call(dst=(ctypes.c_void_p * 1)(0x1000400)))       # inside M
    call(n=0)
    ids = (ctypes.c_uint32 * 9)(*[5] * 9)
    slots = (ctypes.c_void_p * 2)(0x100000, 0x200000)
    lin = lambda n=1, task_ids=ids, group=64, layer=0, x=0x300000, xd=0, xs=128, pb=0x400000, pm=slots, y=0x500000, yd=0, ys=32, ws=None, wn=0: \
        randes.randes_packed_linear_tasks(plan.handle, 1.0, layer, group, task_ids, n, x, xd, xs, pb, pm, y, yd, ys, None, ws, wn)
    _refused(INV, lambda: lin(layer=2))
    _refused(INV, lambda: lin(task_ids=None))
    _refused(randes.UNKNOWN_TASK, lambda: lin(task_ids=(ctypes.c_uint32 * 1)(4)))
    _refused(INV, lambda: lin(pb=None))
    _refused(MIS, lambda: lin(pb=0x400004))
    _refused(INV, lambda: lin(pm=None))
    _refused(INV, lambda: lin(pm=(ctypes.c_void_p * 2)(None, None)))
    _refused(INV, lambda: lin(y=0x400000))
    _refused(INV, lambda: lin(y=0x300000))
    _refused(INV, lambda: lin(xs=100, n=2))
    _refused(DT, lambda: lin(xd=9))
    _refused(WS, lambda: lin(n=9))
    _refused(WS, lambda: lin(n=9, ws=0x600000, wn=100))
    lin(n=0)
    plan.close()
    gauss = randes.Plan([32], [128], [0], [randes.GAUSS], task_ids=[5], seeds=[1], host_only=True)
    _refused(INV, lambda: randes.randes_retrieve_packed(gauss.handle, 5, 1.0, layers, 1, base, 0x1000000, 64, to, None))
    gauss.close()


def test_score_arguments():
    z, t, o = 0x10000, 0x20000, 0x30000
    call = lambda z=z, dt=0, n=4, v=100, s=100, t=t, scale=1.0, k=0, lp=o, h=o + 64, st=o + 128, ids=None, tops=None: \
        randes.randes_token_scores(z, dt, n, v, s, t, scale, k, lp, h, st, ids, tops, None)
    _refused(DT, lambda: call(dt=2))
    for scale in (0.0, -1.0, float("nan"), float("inf"), 1e-9):
        _refused(INV, lambda: call(scale=scale))
    _refused(INV, lambda: call(k=65, ids=o, tops=o))
    _refused(INV, lambda: call(k=1))
    _refused(INV, lambda: call(lp=None))
    _refused(INV, lambda: call(h=None))
    _refused(INV, lambda: call(z=None))
    _refused(INV, lambda: call(s=99))
    _refused(MIS, lambda: call(z=z + 2))
    _refused(MIS, lambda: call(t=t + 4))
    _refused(MIS, lambda: call(h=o + 2))
    _refused(INV, lambda: call(v=0x80000000, s=0x80000000))
    call(n=0)
    back = lambda t=t, g=o, grad=0x40000, gs=100, st=o + 128: \
        randes.randes_token_scores_backward(z, 0, 4, 100, 100, t, 1.0, st, o + 64, g, None, grad, gs, None)
    _refused(INV, lambda: back(t=None))
    _refused(INV, lambda: back(grad=None))
    _refused(INV, lambda: back(gs=50))
    _refused(INV, lambda: back(st=None))
    _refused(INV, lambda: back(grad=z + 400))                               # the logits one row further


def test_sizes_next_to_the_end_of_32_bits_are_refused():
    """Rows and columns are rounded up to whole records in 32 bits."""
    arr = lambda *a: (ctypes.c_void_p * len(a))(*a)
    for rows, cols in ((1, 0xFFFFFFFF), (1, 0xFFFFFF81), (0xFFFFFFFF, 1), (0xFFFFFFC1, 1)):
        assert randes.randes_packed_bytes(rows, cols, 64) == 0
        m = (randes.Matrix * 1)((0x10000, rows, cols, cols))
        for dtype in (randes.F32, randes.BF16):
            _refused(INV, lambda: randes.randes_pack(m, 1, dtype, 64, arr(0x1000000000000), None))
            _refused(INV, lambda: randes.randes_unpack(arr(0x1000000000000), 1, 64, m, dtype, None))
        _refused(INV, lambda: randes.randes_packed_linear(0x1000000000000, rows, cols, 64, 0x10000, 0, cols, 1, 0x2000000000000, 0, rows, None))
    for rows, cols in ((1, 0xFFFFFF00), (0xFFFFFF00, 1), (65535, 65537)):
        assert randes.randes_packed_bytes(rows, cols, 128) == -(-rows // 64) * -(-cols // 128) * 4224
