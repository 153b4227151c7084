"""Matrices in eight bits against the definition in fp64 on the same inputs, and products of them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import randes_oracle as ro                     # noqa: E402
from paper_2505_11204_b200 import build, randes            # noqa: E402

TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def eight(v):
    """What eight bits keep of a matrix, in fp64: every block of 128 columns against the least power of two, 2^-100 at least, that takes its
    greatest magnitude to 448; three bits behind the leading one, steps of 2^-9 below 2^-6."""
    rows, cols = v.shape
    b = torch.nn.functional.pad(v.double(), (0, -cols % 128)).view(rows, -1, 128)
    top = b.abs().amax(2, keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(top == 0, torch.full_like(e, -100), e).clamp(min=-100)
    unit = torch.ldexp(torch.ones_like(top), e)
    t = b / unit
    _, te = torch.frexp(t)
    step = torch.ldexp(torch.ones_like(t), (te - 1).clamp(min=-6) - 3)
    q = torch.round(t / step) * step * unit
    q = torch.where(torch.isfinite(top), q, torch.full_like(q, float("nan")))
    return q.view(rows, -1)[:, :cols]


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double(), nan=7.25), torch.nan_to_num(b.double(), nan=7.25))


def weight(rows, cols, dtype, seed=0, scale=0.02):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(rows, cols, generator=gen, device="cuda") * scale
    w *= torch.exp2(torch.randint(-14, 3, w.shape, generator=gen, device="cuda").float())      # codes of every size
    return w.to(dtype)


SHAPES = [(1, 1), (1, 128), (3, 127), (5, 129), (128, 128), (130, 257), (127, 512), (16, 640), (200, 1000), (257, 2049), (1, 8193), (1030, 8), (640, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_pack_and_unpack(shape, dtype):
    w = weight(*shape, dtype)
    p = randes.pack8(w)
    want = eight(w)
    for code, t in ((randes.F32, torch.float32), (randes.BF16, torch.bfloat16)):
        got = p.unpack(out_dtype=code)
        assert got.dtype is t and same(got, want)          # at most four significant bits: exact in either type
    assert p.nbytes == randes.randes_packed_eight_bytes(*shape)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,first", [(1, 0), (8, 0), (0, 3), (5, 1), (64, 16)])
def test_strided_rows_and_any_alignment(dtype, pad, first):
    rows, cols = 37, 300
    buf = weight(rows, cols + pad + first, dtype)
    w = buf[:, first:first + cols]
    assert same(randes.pack8(w).unpack(), eight(w))
    assert same(randes.pack8_transposed(w).unpack(), eight(w.t()))
    out = torch.full((rows, cols + pad + first), -3.0, dtype=dtype, device="cuda")
    randes.pack8(w).unpack(out=out[:, first:first + cols])
    assert same(out[:, first:first + cols], eight(w))
    assert (out[:, :first] == -3).all() and (out[:, first + cols:] == -3).all()      # what lies between the rows is left alone


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_transposed_and_both(shape, dtype):
    w = weight(*shape, dtype, 1)
    t = randes.pack8_transposed(w)
    assert (t.rows, t.cols) == (shape[1], shape[0]) and same(t.unpack(), eight(w.t()))
    p, t2 = randes.pack8_both(w)
    assert same(p.unpack(), eight(w)) and same(t2.unpack(), t.unpack())
    kept = randes.pack8_transposed(p)                      # the transpose of what was kept
    assert same(kept.unpack(), eight(eight(w).t()))


def test_values_survive_the_change_of_blocks():
    w = weight(300, 500, torch.float32, 2)
    w = torch.where(w.abs() < 2.0 ** -9, torch.zeros_like(w), w).clamp(-0.25, 0.25)      # within 2^7 of one another: subnormal in no block
    p = randes.pack8(w)
    assert torch.equal(randes.pack8_transposed(p).unpack().t(), p.unpack())


def test_values_at_the_borders():
    big = torch.finfo(torch.float32).max
    rows = [[448.0], [448.0001], [449.0], [896.0], [896.1], [1.75, 1.0], [1.7500001, 1.0], [big, 1.0, -big], [2.0 ** -91, 2.0 ** -100, 2.0 ** -110],
            [2.0 ** -92 * 1.75, 2.0 ** -101], [1e-40, -1e-45], [0.0], [-0.0, 0.0], [464.0, 1.0625, 1.1875, 2.0 ** -9, 3 * 2.0 ** -10, 2.0 ** -10, 1.01 * 2.0 ** -10]]
    w = torch.zeros(len(rows), 130, device="cuda")
    for i, r in enumerate(rows):
        w[i, :len(r)] = torch.tensor(r)
    # fp32's greatest number is (2 - 2^-23) 2^127 = 255.99.. * 2^120: its code is 256, and 256 * 2^120 = 2^128 is an infinity in fp32
    want = eight(w).float()
    assert torch.isinf(want[7, 0]) and torch.isinf(want[7, 2]) and torch.isinf(want).sum() == 2
    assert same(randes.pack8(w).unpack(), want)
    assert same(randes.pack8_both(w)[0].unpack(), want)
    assert same(randes.pack8_transposed(w.t().contiguous()).unpack(), want)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_block_that_is_not_finite_reads_back_as_nan(bad):
    for dtype in TYPES:
        w = weight(140, 300, dtype, 3)
        w[2, 5] = w[139, 299] = bad
        got = randes.pack8(w).unpack()
        assert same(got, eight(w)) and torch.isnan(got[2, :128]).all() and torch.isfinite(got[2, 128:]).all() and torch.isnan(got[139, 256:]).all()
        p, t = randes.pack8_both(w)
        assert same(p.unpack(), eight(w)) and same(t.unpack(), eight(w.t()))
        assert torch.isnan(randes.pack8_transposed(p).unpack()[5, :128]).all()


def test_lists_empty_matrices_and_one_launch_per_32():
    ws = [weight(10 + i, 20 * i, torch.bfloat16, i) for i in range(40)]      # (the first has no columns)
    before = randes.randes_launch_count()
    ps = randes.pack8(ws)
    assert randes.randes_launch_count() - before == 2
    assert all(same(p.unpack(), eight(w)) for p, w in zip(ps[1:], ws[1:]))
    assert ps[0].unpack().shape == (10, 0) and randes.pack8([]) == []
    e = randes.pack8_transposed(torch.empty(0, 5, device="cuda"))
    assert (e.rows, e.cols) == (5, 0) and randes.pack8_transposed(randes.pack8(torch.empty(3, 0, device="cuda"))).unpack().shape == (0, 3)


@pytest.mark.parametrize("storage,m_dtype", [(0, 0), (1, 0), (1, 1)])
@pytest.mark.parametrize("flags", [randes.SHUFFLE | randes.FLIP, randes.FLIP, randes.SHUFFLE, 0])
def test_retrieve_packed8_is_the_packed_retrieved_weight(storage, m_dtype, flags):
    rows, cols = [33, 33, 33, 5, 70], [200, 200, 200, 130, 512]
    dt, mt = TYPES[storage], TYPES[m_dtype]
    plan = randes.Plan(rows, cols, [0, 0, 0, 1, 2], [flags, flags, flags], storage=storage, m_dtype=m_dtype, task_ids=[3, 9], seeds=[5, 6])
    base = [weight(r, c, dt, i) for i, (r, c) in enumerate(zip(rows, cols))]
    models = [[weight(r, c, dt, 10 * t + i) for i, (r, c) in enumerate(zip(rows, cols))] for t in (1, 2)]
    M = plan.compress(base, models)
    assert M.dtype is mt
    got = plan.retrieve_packed8(9, 0.4, base, M)
    want = plan.retrieve(9, 0.4, base, M)
    assert all(same(g.unpack(), eight(w)) for g, w in zip(got, want))
    some = plan.retrieve_packed8(9, 0.4, base, M, layers=[4, 1])
    assert torch.equal(some[0].unpack(), got[4].unpack()) and torch.equal(some[1].unpack(), got[1].unpack())
    plan.close()


# ---- products ---------------------------------------------------------------------------------
def bound(x, w):
    """Sums of exact products in fp32: a step of 32 columns adds its products and the sum so far, all cut at 2^-23 of the greatest at worst
    (34 summands), and there are cols / 32 steps; no partial sum is beyond the sum of magnitudes.  Up to 8 partial sums of that kind
    are added in fp32 at the end."""
    return (x.shape[1] / 32 + 34 + 8) * 2.0 ** -23 * (x.abs() @ w.abs().t())


PRODUCTS = [(1, 1, 1), (1, 128, 128), (1, 4096, 1024), (2, 130, 500), (7, 70, 127), (16, 128, 129), (17, 300, 640), (32, 257, 513), (33, 1000, 256),
            (48, 511, 768), (64, 1, 1000), (65, 130, 2049), (100, 700, 384), (128, 128, 4096), (129, 129, 129), (200, 1025, 1500), (257, 260, 512),
            (513, 400, 100), (1000, 4096, 1024), (300, 20000, 130)]


@pytest.mark.parametrize("y_dtype", [randes.F32, randes.BF16])
@pytest.mark.parametrize("tokens,rows,cols", PRODUCTS)
def test_products(tokens, rows, cols, y_dtype):
    x8, w8 = randes.pack8(weight(tokens, cols, torch.bfloat16, 1, 1.0)), randes.pack8(weight(rows, cols, torch.float32, 2))
    x, w = x8.unpack().double(), w8.unpack().double()
    before = randes.randes_linear_giveups()                # (counts for the life of the process)
    y = randes.packed8_linear(x8, w8, y_dtype=y_dtype)
    want = x @ w.t()
    tol = bound(x, w) + (2.0 ** -8 * want.abs() if y_dtype else 0)
    assert y.shape == (tokens, rows) and ((y.double() - want).abs() <= tol).all()
    assert torch.equal(randes.packed8_linear(x8, w8, y_dtype=y_dtype), y)      # the same again, bit for bit
    assert randes.randes_linear_giveups() == before


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,rows,cols", [(1, 50, 1), (1, 4096, 1024), (1, 300, 129), (3, 130, 700), (9, 1000, 2050), (16, 128, 4096), (16, 20000, 520), (17, 200, 300),
                                              (20, 50, 300), (200, 300, 400)])
def test_a_tensor_is_packed_on_the_way(tokens, rows, cols, dtype):
    w = randes.pack8(weight(rows, cols, torch.bfloat16))
    for pad, first in ((0, 0), (3, 1), (8, 8)):
        x = weight(tokens, cols + pad + first, dtype, 1, 1.0)[:, first:first + cols]
        if tokens > 1 and cols > 128:
            x[1, 3], x[0, cols - 1] = float("nan"), 0.0
        a, b = randes.packed8_linear(x, w), randes.packed8_linear(randes.pack8(x), w)
        assert same(a, b) and torch.isfinite(a[0]).all()


@pytest.mark.parametrize("tokens", [1, 20, 150])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_between_and_behind_are_left_alone(tokens, dtype):
    rows, cols = 131, 260
    x8, w8 = randes.pack8(weight(tokens, cols, dtype, 1, 1.0)), randes.pack8(weight(rows, cols, dtype, 2))
    out = torch.full((tokens + 2, rows + 3), -3.0, dtype=dtype, device="cuda")
    y = out[1:1 + tokens, 1:1 + rows]
    randes.packed8_linear(x8, w8, y=y)
    assert torch.equal(y, randes.packed8_linear(x8, w8, y_dtype=int(dtype is torch.bfloat16)))
    out[1:1 + tokens, 1:1 + rows] = -3
    assert (out == -3).all()


def test_products_with_blocks_that_are_not_finite_and_of_extreme_scales():
    x, w = weight(30, 600, torch.float32, 1, 1.0), weight(200, 600, torch.float32, 2)
    x[4, 130], w[17, 599] = float("nan"), float("inf")
    y = randes.packed8_linear(x, randes.pack8(w))
    bad = torch.isnan(y)
    assert bad[4].all() and bad[:, 17].all() and bad.sum() == 30 + 200 - 1
    # scales at both ends of their range: 2^-100 and 2^119 units, a sum that leaves fp32
    x, w = torch.zeros(3, 256, device="cuda"), torch.zeros(5, 256, device="cuda")
    x[0], x[1], x[2] = 2.0 ** 120, 2.0 ** -95, 2.0 ** 127
    w[0], w[1], w[2], w[3], w[4] = 2.0 ** -95, 2.0 ** 100, 2.0 ** -20, 0.0, 2.0 ** 127
    y, want = randes.packed8_linear(x, randes.pack8(w)).double(), eight(x) @ eight(w).t()
    size = want.abs()
    fits = (size < 2.0 ** 128) & (size >= 2.0 ** -126)
    assert torch.equal(y[fits], want[fits]) and torch.isinf(y[size >= 2.0 ** 128]).all() and (y[size < 2.0 ** -126].abs() < 2.0 ** -126).all()


def test_products_over_no_columns_and_of_no_tokens():
    x, w = randes.pack8(torch.empty(4, 0, device="cuda")), randes.pack8(torch.empty(6, 0, device="cuda"))
    y = torch.full((4, 8), -3.0, device="cuda")
    randes.packed8_linear(x, w, y=y[:, :6])
    assert (y[:, :6] == 0).all() and (y[:, 6:] == -3).all()
    assert randes.packed8_linear(torch.empty(0, 40, device="cuda"), randes.pack8(torch.ones(6, 40, device="cuda"))).shape == (0, 6)


def test_gradients_of_a_layer_out_of_checkpoints():
    n, rows, cols = 300, 200, 500
    x, w, g = weight(n, cols, torch.bfloat16, 1, 1.0), weight(rows, cols, torch.float32, 2), weight(n, rows, torch.bfloat16, 3)
    kept = randes.pack8(x)
    g8, g8t = randes.pack8_both(g)
    dx = randes.packed8_linear(g8, randes.pack8_transposed(w))
    dw = randes.packed8_linear(g8t, randes.pack8_transposed(kept))
    a, b = eight(g), eight(w.t())
    assert ((dx.double() - a @ b.t()).abs() <= bound(a, b)).all()
    a, b = eight(g.t()), eight(eight(x).t())
    assert ((dw.double() - a @ b.t()).abs() <= bound(a, b)).all()


def test_side_stream_and_graph():
    x, w8 = weight(5, 700, torch.bfloat16, 1, 1.0), randes.pack8(weight(900, 700, torch.bfloat16, 2))
    want = randes.packed8_linear(x, w8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = randes.packed8_linear(x, w8)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    g, out, buf = torch.cuda.CUDAGraph(), torch.empty_like(want), x.clone()
    with torch.cuda.graph(g):
        randes.packed8_linear(buf, w8, y=out)
    for seed in (4, 5):
        buf.copy_(weight(5, 700, torch.bfloat16, seed, 1.0))
        g.replay()
        assert torch.equal(out, randes.packed8_linear(buf, w8))


def test_refusals():
    x, w = torch.zeros(4, 256, device="cuda"), randes.pack8(torch.zeros(8, 256, device="cuda"))
    x8 = randes.pack8(x)
    y = torch.empty(4, 8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    call = lambda wa=w.address, xa=x8.address, ya=y, ydt=0, st=8, n=4, rows=8, cols=256: randes.randes_packed_eight_linear(wa, rows, cols, xa, n, ya, ydt, st, s)
    inv, mis = randes.INVALID_ARGUMENT, randes.MISALIGNED
    many = torch.zeros(400, 256, device="cuda")
    typed = lambda xa, n=4, dt=0, st=256, ws=None: randes.randes_packed_eight_linear(w.address, 8, 256, xa, n, y if n <= 4 else out, 0, 8, s, dt, st, ws, 1 << 17 if ws is not None else 0)
    out = torch.empty(17, 8, device="cuda")
    inside = torch.empty(w.data.numel(), dtype=torch.uint8, device="cuda")
    cases = [(lambda: call(wa=None), inv), (lambda: call(xa=None), inv), (lambda: call(ya=None), inv), (lambda: call(wa=w.address + 8), mis),
             (lambda: call(xa=x8.address + 4), mis), (lambda: call(ya=y.data_ptr() + 2), mis), (lambda: call(st=7), inv), (lambda: call(ydt=2), randes.UNSUPPORTED_DTYPE),
             (lambda: call(n=0xFFFFFFFF), inv), (lambda: call(ya=w.data), inv), (lambda: call(ya=x8.data), inv),
             (lambda: randes.pack8(x.double()), randes.UNSUPPORTED_DTYPE), (lambda: randes.pack8(x.t()), inv), (lambda: randes.pack8(x.cpu()), inv),
             (lambda: randes.pack8([x, x.bfloat16()]), inv), (lambda: randes.packed8_linear(x[:, :200], w), inv), (lambda: randes.packed8_linear(x, x), inv),
             (lambda: randes.packed8_linear(x, w, y=y.t()), inv), (lambda: randes.Packed8Matrix(200, 256, inside), inv),
             (lambda: randes.Packed8Matrix(8, 100, inside[8:]), mis), (lambda: randes.Packed8Matrix(8, 100, inside.cpu()), inv),
             (lambda: w.unpack(out=torch.empty(8, 255, device="cuda")), inv),
             (lambda: randes.randes_transpose_eight(w.address, 8, 256, w.address, s), inv), (lambda: typed(x, st=255), inv), (lambda: typed(x.data_ptr() + 2), mis),
             (lambda: typed(x, dt=3), randes.UNSUPPORTED_DTYPE), (lambda: typed(y, n=1), inv), (lambda: typed(many, n=17), randes.WORKSPACE_TOO_SMALL),
             (lambda: typed(many, n=17, ws=many), inv)]
    for i, (f, code) in enumerate(cases):
        with pytest.raises(randes.RandesError) as e:
            f()
        assert e.value.code == code, (i, e.value)
    again = randes.Packed8Matrix(8, 256, w.data.clone())
    assert torch.equal(again.unpack(), w.unpack())


def test_chains_of_calls_in_graphs_that_fork_and_join():
    """Kernels take their places early: what they read has to be complete all the same, in a captured chain too."""
    n, cols = 64, 1024
    w = [randes.pack8(weight(cols, cols, torch.bfloat16, i)) for i in range(4)]
    x, gain = weight(n, cols, torch.bfloat16, 9, 1.0), torch.ones(cols, device="cuda")

    def chain(x, join):
        h = x
        for q in w:
            f = randes.rms_norm(randes.packed8_linear(h, q, y_dtype=randes.BF16), gain, h, packed=True)
            h = f.h + 0                                    # another library's kernel in between
            if join is not None:
                join[0].wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(join[0]):
                    side = randes.packed8_linear(f.y, q, y_dtype=randes.BF16)
                torch.cuda.current_stream().wait_stream(join[0])
            else:
                side = randes.packed8_linear(f.y, q, y_dtype=randes.BF16)
            h = randes.rms_norm(h, gain, side).h
        return h

    want = chain(x, None)
    torch.cuda.synchronize()
    assert torch.isfinite(want.float()).all()
    for join in (None, [torch.cuda.Stream()]):
        buf, g = x.clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = chain(buf, join)
        for _ in range(5):
            out.zero_()
            g.replay()
            assert torch.equal(out, want)


def test_retrieving_or_turning_may_be_the_first_call(monkeypatch):
    w = torch.randn(130, 300, device="cuda")
    p, t = randes.pack8_both(w)
    plan = randes.Plan([130], [300], [0], [0], task_ids=[0], seeds=[1])
    M = plan.new_superposition()
    M.zero_()
    for first in (lambda: randes.pack8_transposed(randes.Packed8Matrix(130, 300, p.data)), lambda: plan.retrieve_packed8(0, 0.3, [w], M)[0], lambda: p,
                  lambda: randes.packed8_linear(p, p)):
        monkeypatch.setattr(randes, "_torch", None)
        got = first()
        if isinstance(got, randes.Packed8Matrix):
            assert torch.equal(got.unpack(), (t if got.rows == 300 else p).unpack())
    plan.close()
