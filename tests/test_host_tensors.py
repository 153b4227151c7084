"""The calls on torch tensors, without a GPU: tensors that only say where they are, and a library that only notes which device
is current when it is called."""
import contextlib
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2505_11204_b200 import build, randes    # noqa: E402


class Fake:
    """What the binding asks of a CUDA tensor."""

    def __init__(self, shape, dtype=torch.float32, device=0, stride=None, address=0x10000000):
        self.shape, self.dtype, self.device, self.is_cuda, self.address = tuple(shape), dtype, torch.device("cuda", device), True, address
        self._stride = stride or tuple(int(torch.tensor(self.shape[i + 1:]).prod()) for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self._stride

    def data_ptr(self):
        return self.address

    def numel(self):
        return int(torch.tensor(self.shape).prod())

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return self._stride == Fake(self.shape)._stride

    def __getitem__(self, row):      # a row of the statistics
        return Fake(self.shape[1:], self.dtype, self.device.index)


class Library:
    """The real library for what runs on the host alone; the rest notes the current device."""

    LAUNCHING = ("randes_pack", "randes_unpack", "randes_retrieve_packed", "randes_packed_linear", "randes_packed_linear_tasks",
                 "randes_token_scores", "randes_token_scores_backward")

    def __init__(self, real, current):
        self.real, self.current, self.calls = real, current, []

    def __getattr__(self, name):
        if name not in self.LAUNCHING:
            return getattr(self.real, name)

        def noted(*args):
            self.calls.append((name, self.current[0], args))
            return 0
        return noted


@pytest.fixture
def fake(monkeypatch):
    build.build_library()
    current = [0]

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], d if isinstance(d, int) else d.index
        yield
        current[0] = before

    library = Library(randes.lib(), current)
    monkeypatch.setattr(randes, "lib", lambda: library)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index)
    monkeypatch.setattr(torch, "empty", lambda *shape, dtype=torch.float32, device=None: Fake(shape, dtype, torch.device(device).index))
    return library


def _plan(**kw):
    return randes.Plan([64, 64], [128, 128], [0, 0], [randes.SHUFFLE | randes.FLIP], task_ids=[5], seeds=[1], host_only=True, **kw)


def _refused(code, fn):
    with pytest.raises(randes.RandesError) as e:
        fn()
    assert e.value.code == code, (e.value.code, str(e.value))


@pytest.mark.parametrize("where", [0, 1, 3])
def test_the_library_runs_with_the_tensors_device_current(fake, where):
    w, x = Fake((64, 128), device=where), Fake((3, 128), torch.bfloat16, where)
    p = randes.pack(w)
    packed = randes.pack([w, w])
    p.unpack()
    randes.packed_linear(x, p)
    randes.packed_linear(Fake((12, 128), device=where), p)      # with a workspace
    plan = _plan()
    M = Fake((plan.m_bytes // 4,), device=where)
    plan.retrieve_packed(5, 1.0, [w, w], M)
    plan.packed_linear([5, 5, 5], 1.0, 0, x, p, packed)
    z, t, g = Fake((3, 100), device=where), Fake((3,), torch.int64, where), Fake((3,), device=where)
    r = randes.token_scores(z, t, top_k=4)
    randes.token_scores_backward(z, t, r, g, g)
    assert [c[0] for c in fake.calls] == ["randes_pack", "randes_pack", "randes_unpack", "randes_packed_linear", "randes_packed_linear",
                                          "randes_retrieve_packed", "randes_packed_linear_tasks", "randes_token_scores",
                                          "randes_token_scores_backward"]
    for name, current, args in fake.calls:
        assert current == where, name
        assert args[-1] == 1000 + where, "%s: stream" % name
    assert fake.current[0] == 0                                 # as the caller left it
    plan.close()


def test_the_callers_device_comes_back_after_an_error(fake):
    failing = lambda *a: 7
    with pytest.raises(randes.RandesError):
        randes._call(torch.device("cuda", 2), failing)
    assert fake.current[0] == 0


def test_tensors_of_two_devices_are_refused(fake):
    inv = randes.INVALID_ARGUMENT
    w, other = Fake((64, 128)), Fake((64, 128), device=1)
    p, q = randes.pack(w), randes.pack(other)
    x, y = Fake((3, 128)), Fake((3, 64))
    plan = _plan()
    del fake.calls[:]
    _refused(inv, lambda: randes.pack([w, other]))
    _refused(inv, lambda: p.unpack(out=other))
    _refused(inv, lambda: randes.packed_linear(x, q))
    _refused(inv, lambda: randes.packed_linear(x, p, y=Fake((3, 64), device=1)))
    _refused(inv, lambda: plan.packed_linear([5] * 3, 1.0, 0, x, q, [p, p]))
    _refused(inv, lambda: plan.packed_linear([5] * 3, 1.0, 0, x, p, [p, q]))
    _refused(inv, lambda: plan.packed_linear([5] * 3, 1.0, 0, x, p, [p, p], y=Fake((3, 64), device=1)))
    z, t, g = Fake((3, 100)), Fake((3,), torch.int64), Fake((3,))
    _refused(inv, lambda: randes.token_scores(z, Fake((3,), torch.int64, 1)))
    r = randes.token_scores(z, t)
    _refused(inv, lambda: randes.token_scores_backward(Fake((3, 100), device=1), Fake((3,), torch.int64, 1), r, None))
    _refused(inv, lambda: randes.token_scores_backward(z, t, r, Fake((3,), device=1)))
    _refused(inv, lambda: randes.token_scores_backward(z, t, r, g, out=Fake((3, 100), device=1)))
    assert [c[0] for c in fake.calls] == ["randes_token_scores"]
    randes.packed_linear(x, p, y=y)
    plan.packed_linear([5] * 3, 1.0, 0, x, p, [p, None])
    plan.close()


def test_slots_are_packed_matrices_not_addresses(fake):
    """An array of addresses says neither how many slots it names nor what they hold."""
    p, x, plan = randes.pack(Fake((64, 128))), Fake((2, 128)), _plan()
    for n in (1, 2, 5):
        _refused(randes.INVALID_ARGUMENT, lambda: plan.packed_linear([5, 5], 1.0, 0, x, p, (ctypes.c_void_p * n)(*[p.address] * n)))
    _refused(randes.INVALID_ARGUMENT, lambda: plan.packed_linear([5, 5], 1.0, 0, x, p, [p, p.address]))
    _refused(randes.INVALID_ARGUMENT, lambda: plan.packed_linear([5, 5], 1.0, 0, x, p.address, [p, p]))
    plan.packed_linear([5, 5], 1.0, 0, x, p, (p, p))
    plan.close()


def test_task_ids_of_any_integer_array_are_read_as_numbers(fake):
    p, x, plan = randes.pack(Fake((64, 128))), Fake((3, 128)), _plan()
    for ids in ([5, 6, 7], (5, 6, 7), (ctypes.c_uint32 * 3)(5, 6, 7), (ctypes.c_uint8 * 3)(5, 6, 7), (ctypes.c_uint64 * 3)(5, 6, 7),
                torch.tensor([5, 6, 7])):
        plan.packed_linear(ids, 1.0, 0, x, p, [p, p])
        passed = fake.calls[-1][2][4]
        assert passed._type_ is ctypes.c_uint32 and list(passed) == [5, 6, 7], type(ids)
    plan.close()


def test_a_packed_matrix_checks_the_buffer_it_is_made_of(fake):
    inv = randes.INVALID_ARGUMENT
    need = randes.randes_packed_bytes(64, 128, 64)
    buffer = lambda n, **kw: Fake((n,), kw.pop("dtype", torch.uint8), **kw)
    p = randes.PackedMatrix(64, 128, 64, buffer(need))           # as read back from a file
    assert p.nbytes == need and randes.pack(Fake((64, 128))).nbytes == need
    randes.PackedMatrix(64, 128, 64, buffer(need + 16))
    randes.PackedMatrix(0, 128, 64, buffer(0))
    randes.PackedMatrix(64, 128, 64, buffer(need // 4, dtype=torch.int32))
    _refused(inv, lambda: randes.PackedMatrix(64, 128, 64, buffer(need - 1)))
    _refused(inv, lambda: randes.PackedMatrix(64, 128, 32, buffer(need)))
    _refused(inv, lambda: randes.PackedMatrix(65, 128, 64, buffer(need)))
    _refused(inv, lambda: randes.PackedMatrix(64, 128, 48, buffer(need)))
    _refused(inv, lambda: randes.PackedMatrix(70000, 70000, 64, buffer(need)))
    _refused(inv, lambda: randes.PackedMatrix(64, 128, 64, buffer(need, stride=(2,))))
    _refused(inv, lambda: randes.PackedMatrix(64, 128, 64, torch.zeros(need, dtype=torch.uint8)))       # host memory
    _refused(randes.MISALIGNED, lambda: randes.PackedMatrix(64, 128, 64, buffer(need, address=0x10000008)))


@pytest.mark.parametrize("storage,m_dtype", [(randes.F32, randes.F32), (randes.BF16, randes.F32), (randes.F32, randes.BF16)])
def test_retrieve_packed_checks_the_weights_and_the_superposition(fake, storage, m_dtype):
    inv, dt = randes.INVALID_ARGUMENT, randes.UNSUPPORTED_DTYPE
    types = {randes.F32: torch.float32, randes.BF16: torch.bfloat16}
    wt, mt, wrong = types[storage], types[m_dtype], {torch.float32: torch.bfloat16, torch.bfloat16: torch.float32}
    plan = _plan(storage=storage, m_dtype=m_dtype)
    n = plan.m_bytes // mt.itemsize
    w, M = Fake((64, 128), wt), Fake((n,), mt)
    call = lambda base=(w, w), m=M, **kw: plan.retrieve_packed(5, 1.0, base, m, **kw)
    _refused(dt, lambda: call((w, Fake((64, 128), wrong[wt]))))
    _refused(dt, lambda: call((Fake((64, 128), torch.float16), w)))
    _refused(inv, lambda: call((w, Fake((64, 128), wt, stride=(136, 1)))))     # rows apart: the library reads them as dense
    _refused(inv, lambda: call((w, Fake((128, 64), wt))))
    _refused(inv, lambda: call((w, Fake((64, 127), wt))))
    _refused(inv, lambda: call((w, Fake((64, 128), wt, device=1))))
    _refused(inv, lambda: call((w, torch.zeros(64, 128, dtype=wt))))           # host memory
    _refused(inv, lambda: call((w, None)))
    _refused(inv, lambda: call((w,)))
    _refused(inv, lambda: call((w,), layers=[1]))
    _refused(inv, lambda: call((ctypes.c_void_p * 1)(0x10000)))
    _refused(inv, lambda: call((ctypes.c_uint32 * 2)(0x10000, 0x20000)))
    _refused(dt, lambda: call(m=Fake((2 * n,), wrong[mt])))
    _refused(inv, lambda: call(m=Fake((n - 1,), mt)))
    _refused(inv, lambda: call(m=Fake((n,), mt, stride=(2,))))
    _refused(inv, lambda: call(m=torch.zeros(n, dtype=mt)))
    _refused(dt, lambda: plan.pack_superposition(Fake((2 * n,), wrong[mt])))
    _refused(inv, lambda: plan.pack_superposition(Fake((n - 1,), mt)))
    assert not fake.calls
    call()
    call((w,), layers=[0])                                                     # only the named ones are read
    call((w, None), layers=[0])
    call((Fake((64 * 128,), wt), Fake((64, 2, 64), wt)))
    call((ctypes.c_void_p * 2)(0x10000, 0x20000))                              # addresses, as the other methods take them
    call((), layers=[])
    assert len(fake.calls) == 6
    plan.close()
