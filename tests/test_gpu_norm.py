"""The norm with the residual's addition and its gradient against the formulas in fp64."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2505_11204_b200 import build, randes            # noqa: E402

TYPES = [torch.float32, torch.bfloat16]
EPS = 1e-6
# fp32: a thread adds up to 32 squares, 5 + 31 further sums behind it; half of that error reaches the root; three roundings
FP32 = (32 + 36) / 2 * 2.0 ** -24 + 4 * 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def rows_of(n, cols, dtype, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, cols, generator=gen, device="cuda") * scale).to(dtype)


def step(dtype):
    return torch.finfo(dtype).eps / 2


def norm64(h, gain):
    h = h.double()
    rstd = 1 / torch.sqrt((h * h).mean(1) + EPS)
    return rstd, h * rstd[:, None] * (1 if gain is None else gain.double())


def check_eight(p, y, rel):
    """A code is off by half a step: 2^-4 of the value, or 2^-10 of the block's unit; the unit follows the greatest value, which may have
    come out `rel` larger or smaller and may then be twice what it is for y."""
    rows, cols = y.shape
    pad = torch.nn.functional.pad(y, (0, -cols % 128)).view(rows, -1, 128)
    unit = 2 * torch.exp2(torch.ceil(torch.log2(pad.abs().amax(2, keepdim=True).clamp(min=1e-30) / 448)))
    tol = ((2.0 ** -4 + 2 * rel) * pad.abs() + 2.0 ** -10 * unit).flatten(1)[:, :cols]
    assert ((p.unpack().double() - y).abs() <= tol).all()


SHAPES = [(1, 1), (1, 1024), (3, 7), (5, 127), (130, 128), (9, 129), (6, 256), (33, 300), (7, 513), (4, 1000), (4, 1024), (5, 1025), (3, 2048), (2, 2056), (3, 4001),
          (2, 4096), (3, 6000), (2, 8192), (2, 9001), (1, 16384), (2, 16392), (1, 32768), (500, 64), (7, 64), (5, 768), (3, 640), (9, 256), (3, 12345)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,cols", SHAPES)
def test_forward(n, cols, dtype):
    x, r, gain = rows_of(n, cols, dtype, 1), rows_of(n, cols, dtype, 2, 3.0), 1 + 0.3 * rows_of(1, cols, torch.float32, 3)[0]
    f = randes.rms_norm(x, gain, r, eps=EPS)
    h = (x.float() + r.float()).to(dtype)
    rstd, y = norm64(h, gain)
    assert torch.equal(f.h, h) and f.kept is None
    assert ((f.rstd.double() - rstd).abs() <= FP32 * rstd).all()
    assert ((f.y.double() - y).abs() <= (FP32 + (step(dtype) if dtype is torch.bfloat16 else 0)) * y.abs()).all()
    p = randes.rms_norm(x, gain, r, eps=EPS, packed=True, checkpoint=True)
    assert torch.equal(p.h, h) and torch.equal(p.rstd, f.rstd)
    check_eight(p.y, y, FP32)
    assert torch.equal(p.kept.unpack(), randes.pack8(h).unpack())      # the checkpoint is the stored residual's eight bits
    if dtype is torch.float32:
        assert torch.equal(p.y.unpack(), randes.pack8(f.y).unpack())   # and the output that of the norm's own output
    bare = randes.rms_norm(x, None, eps=EPS)
    assert bare.h is x and ((bare.y.double() - norm64(x, None)[1]).abs() <= (FP32 + (step(dtype) if dtype is torch.bfloat16 else 0)) * norm64(x, None)[1].abs()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("n,cols", SHAPES + [(2000, 64), (1500, 1024), (700, 2050), (256, 1024), (200, 768), (40, 5000), (32, 8192)])
def test_backward(n, cols, kept, dtype):
    x, r, gain = rows_of(n, cols, dtype, 1), rows_of(n, cols, dtype, 2, 3.0), 1 + 0.3 * rows_of(1, cols, torch.float32, 3)[0]
    g, gh = rows_of(n, cols, dtype, 4), rows_of(n, cols, dtype, 5)
    f = randes.rms_norm(x, gain, r, eps=EPS, checkpoint=True)
    dx, dgain = randes.rms_norm_backward(g, f.kept if kept else f.h, f.rstd, gain, dh=gh)
    rstd, hd = f.rstd.double()[:, None], (f.kept.unpack() if kept else f.h).double()
    nd, gg = hd * rstd, g.double() * gain.double()
    inner = (gg * nd).mean(1, keepdim=True)
    want = rstd * (gg - nd * inner) + gh.double()
    # the mean's error against the mean of magnitudes; a few roundings of every term
    size = rstd * (gg.abs() + nd.abs() * (gg * nd).abs().mean(1, keepdim=True)) + gh.double().abs()
    assert ((dx.double() - want).abs() <= (2 * FP32 + 4 * 2.0 ** -24) * size + (step(dtype) * want.abs() if dtype is torch.bfloat16 else 0)).all()
    # sums over rows: a CTA or warp adds at most n of them one after the other, then up to 8 + 1184 / 16 + 16 shares
    terms = (g.double() * nd).abs().sum(0)
    assert ((dgain.double() - (g.double() * nd).sum(0)).abs() <= (n + 100) * 2.0 ** -24 * terms).all()
    alone, none = randes.rms_norm_backward(g, f.kept if kept else f.h, f.rstd)
    n1 = hd * rstd
    size = rstd * (g.double().abs() + n1.abs() * (g.double() * n1).abs().mean(1, keepdim=True))
    want = rstd * (g.double() - n1 * (g.double() * n1).mean(1, keepdim=True))
    assert none is None and ((alone.double() - want).abs() <= (2 * FP32 + 4 * 2.0 ** -24) * size + (step(dtype) * want.abs() if dtype is torch.bfloat16 else 0)).all()
    again = randes.rms_norm_backward(g, f.kept if kept else f.h, f.rstd, gain, dh=gh)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgain)


# rows in several parts, more of them than there are clusters for; a last part of one column, of one block, of a whole part
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("n,cols", [(200, 8193), (180, 9216), (90, 12289), (130, 16384), (60, 20481), (50, 28672), (70, 32768)])
def test_backward_of_wide_rows(n, cols, pad, dtype):
    view = lambda seed: rows_of(n, cols + pad, dtype, seed)[:, pad:]
    x, g, gh, gain = view(1), view(2), view(3), 1 + 0.3 * rows_of(1, cols, torch.float32, 4)[0]
    f = randes.rms_norm(x, gain, eps=EPS, checkpoint=True)
    for kept in (False, True):
        hd = (f.kept.unpack() if kept else f.h).double()
        rstd, gd = f.rstd.double()[:, None], g.double()
        nd, gg = hd * rstd, gd * gain.double()
        want = rstd * (gg - nd * (gg * nd).mean(1, keepdim=True)) + gh.double()
        size = rstd * (gg.abs() + nd.abs() * (gg * nd).abs().mean(1, keepdim=True)) + gh.double().abs()
        tol = (2 * FP32 + 4 * 2.0 ** -24) * size + (step(dtype) * want.abs() if dtype is torch.bfloat16 else 0)
        dx, dgain = randes.rms_norm_backward(g, f.kept if kept else f.h, f.rstd, gain, dh=gh)
        assert ((dx.double() - want).abs() <= tol).all()
        # at most n rows one after the other, then the clusters' shares
        assert ((dgain.double() - (gd * nd).sum(0)).abs() <= (n + 100) * 2.0 ** -24 * (gd * nd).abs().sum(0)).all()
        base = rows_of(n, cols + pad, dtype, 2)
        into, _ = randes.rms_norm_backward(base[:, pad:], f.kept if kept else f.h, f.rstd, gain, dh=gh, out=base[:, pad:])
        assert torch.equal(into, dx) and torch.equal(base[:, :pad], rows_of(n, cols + pad, dtype, 2)[:, :pad])


# one width of every number of threads to a row, on 16-byte boundaries and off them
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1281, 1536, 2500, 3064, 4097, 5120, 5121, 6000, 6145, 7168, 7169, 8200, 10241, 12288, 12289, 14336, 14337])
def test_forward_of_every_width(cols, dtype):
    n = 5
    x, r, gain = rows_of(n, cols, dtype, 1), rows_of(n, cols, dtype, 2, 3.0), 1 + 0.3 * rows_of(1, cols, torch.float32, 3)[0]
    p = randes.rms_norm(x, gain, r, eps=EPS, packed=True, checkpoint=True)
    f = randes.rms_norm(x, gain, r, eps=EPS)
    h = (x.float() + r.float()).to(dtype)
    rstd, y = norm64(h, gain)
    assert torch.equal(p.h, h) and torch.equal(f.h, h) and torch.equal(p.rstd, f.rstd)
    assert ((f.rstd.double() - rstd).abs() <= FP32 * rstd).all()
    assert ((f.y.double() - y).abs() <= (FP32 + (step(dtype) if dtype is torch.bfloat16 else 0)) * y.abs()).all()
    check_eight(p.y, y, FP32)
    assert torch.equal(p.kept.unpack(), randes.pack8(h).unpack())


def test_gradient_against_differences():
    n, cols, d = 3, 200, 1e-4
    x, gain, g = rows_of(n, cols, torch.float32, 1), 1 + 0.3 * rows_of(1, cols, torch.float32, 2)[0], rows_of(n, cols, torch.float32, 3)
    loss = lambda h, w: (g.double() * norm64(h, w)[1]).sum()
    f = randes.rms_norm(x, gain, eps=EPS)
    dx, dgain = randes.rms_norm_backward(g, f.h, f.rstd, gain)
    for seed in range(4):
        v, u = rows_of(n, cols, torch.float64, 10 + seed), rows_of(1, cols, torch.float64, 20 + seed)[0]
        num = (loss(x.double() + d * v, gain) - loss(x.double() - d * v, gain)) / (2 * d)
        assert abs(float(num - (dx.double() * v).sum())) <= 1e-4 * float((dx.double() * v).abs().sum())      # d^2 and fp32 are far below
        num = (loss(x, gain.double() + d * u) - loss(x, gain.double() - d * u)) / (2 * d)
        assert abs(float(num - (dgain.double() * u).sum())) <= 1e-4 * float((dgain.double() * u).abs().sum())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,first", [(1, 0), (8, 0), (0, 3), (5, 1), (64, 16)])
def test_strides_and_alignment(dtype, pad, first):
    for n, cols in ((5, 300), (3, 1500)):
        view = lambda seed: rows_of(n, cols + pad + first, dtype, seed)[:, first:first + cols]
        x, r, g, gh = view(1), view(2), view(3), view(4)
        gain = rows_of(1, cols + 1, torch.bfloat16, 5)[0, 1:].contiguous()
        # (rows on 16-byte boundaries are summed in another order than others: either sum is within FP32 of the exact one, so the two are not
        # compared with each other but with the formulas, within the bounds of the tests above)
        h = (x.float() + r.float()).to(dtype)
        rstd, y = norm64(h, gain)
        half = step(dtype) if dtype is torch.bfloat16 else 0
        a = randes.rms_norm(x, gain, r, packed=True, checkpoint=True)
        assert torch.equal(a.h, h) and torch.equal(a.kept.unpack(), randes.pack8(h).unpack()) and ((a.rstd.double() - rstd).abs() <= FP32 * rstd).all()
        check_eight(a.y, y, FP32)
        hb, yb = (torch.full((n, cols + pad + first), -3.0, dtype=dtype, device="cuda") for _ in range(2))
        c = randes.rms_norm(x, gain, r, h=hb[:, first:first + cols], y=yb[:, first:first + cols])
        assert torch.equal(c.h, a.h) and torch.equal(c.rstd, a.rstd) and ((c.y.double() - y).abs() <= (FP32 + half) * y.abs()).all()
        out = torch.full_like(hb, -3.0)
        dx, dgain = randes.rms_norm_backward(g, a.kept, a.rstd, gain, dh=gh, out=out[:, first:first + cols])
        rs = a.rstd.double()[:, None]
        nd, gg = a.kept.unpack().double() * rs, g.double() * gain.double()
        want = rs * (gg - nd * (gg * nd).mean(1, keepdim=True)) + gh.double()
        size = rs * (gg.abs() + nd.abs() * (gg * nd).abs().mean(1, keepdim=True)) + gh.double().abs()
        assert ((dx.double() - want).abs() <= (2 * FP32 + 4 * 2.0 ** -24) * size + half * want.abs()).all()
        assert ((dgain.double() - (g.double() * nd).sum(0)).abs() <= (n + 100) * 2.0 ** -24 * (g.double() * nd).abs().sum(0)).all()
        for buf in (hb, yb, out):
            assert (buf[:, :first] == -3).all() and (buf[:, first + cols:] == -3).all()


@pytest.mark.parametrize("cols", [100, 1111, 4096])
def test_in_place(cols):
    for dtype in TYPES:
        x, r, gain = rows_of(6, cols, dtype, 1), rows_of(6, cols, dtype, 2), rows_of(1, cols, dtype, 3)[0]
        want = randes.rms_norm(x, gain, r)
        a, b = x.clone(), r.clone()
        f = randes.rms_norm(a, gain, b, h=b, y=a)          # the residual is updated, the norm goes where x was
        assert f.h is b and torch.equal(b, want.h) and torch.equal(a, want.y)
        g, gh = rows_of(6, cols, dtype, 4), rows_of(6, cols, dtype, 5)
        grads = randes.rms_norm_backward(g, want.h, want.rstd, gain, dh=gh)
        for which in range(3):
            t = [g.clone(), want.h.clone(), gh.clone()]
            got = randes.rms_norm_backward(t[0], t[1], want.rstd, gain, dh=t[2], out=t[which])
            assert torch.equal(got[0], grads[0]) and torch.equal(got[1], grads[1]) and got[0] is t[which]


def test_extreme_rows():
    x = torch.zeros(6, 300, device="cuda")
    x[1] = 1e30                                            # squares leave fp32
    x[2] = 1e-30                                           # squares vanish: eps is what is left
    x[3, 5], x[4, 7] = float("nan"), float("inf")
    x[5] = torch.finfo(torch.float32).max
    f = randes.rms_norm(x, None, eps=EPS)
    rstd, y = norm64(x, None)
    for r in (0, 1, 2, 5):
        assert ((f.y[r].double() - y[r]).abs() <= FP32 * y[r].abs() + 2.0 ** -149).all()
    assert torch.isnan(f.y[3]).all() and torch.isnan(f.y[4, 7]) and (f.y[4, :7] == 0).all()
    p = randes.rms_norm(x, None, eps=EPS, packed=True)
    assert torch.isnan(p.y.unpack()[3]).all() and torch.isnan(p.y.unpack()[4, :128]).all() and (p.y.unpack()[4, 128:] == 0).all()
    one = randes.rms_norm(x[4:5, :5].clone(), None)        # NaN stops at its row
    assert torch.isfinite(one.y).all()


def test_no_rows_and_graph():
    e = torch.empty(0, 40, device="cuda")
    gain = torch.ones(40, device="cuda")
    f = randes.rms_norm(e, gain, e)
    dx, dgain = randes.rms_norm_backward(e, f.h, f.rstd, gain)
    assert f.y.shape == (0, 40) and dx.shape == (0, 40) and (dgain == 0).all()
    x, r, gain = rows_of(9, 600, torch.bfloat16, 1), rows_of(9, 600, torch.bfloat16, 2), torch.ones(600, device="cuda")
    g = torch.cuda.CUDAGraph()
    randes.rms_norm(x, gain, r)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        f = randes.rms_norm(x, gain, r, packed=True, checkpoint=True)
        dx, dgain = randes.rms_norm_backward(x, f.kept, f.rstd, gain, dh=r)
    for seed in (3, 4):
        x.copy_(rows_of(9, 600, torch.bfloat16, seed))
        g.replay()
        w = randes.rms_norm(x, gain, r, packed=True, checkpoint=True)
        want = randes.rms_norm_backward(x, w.kept, w.rstd, gain, dh=r)
        assert torch.equal(f.y.unpack(), w.y.unpack()) and torch.equal(dx, want[0]) and torch.equal(dgain, want[1])


def test_refusals():
    x, gain = torch.zeros(4, 256, device="cuda"), torch.ones(256, device="cuda")
    f = randes.rms_norm(x, gain, checkpoint=True)
    inv = randes.INVALID_ARGUMENT
    s = torch.cuda.current_stream().cuda_stream
    back = dict(dy=x.data_ptr(), h=x.data_ptr(), rstd=f.rstd.data_ptr(), gain=gain.data_ptr(), dx=f.y.data_ptr(), dgain=gain.data_ptr(), dy_stride=256, h_stride=256,
                dx_stride=256, rows=4, cols=256)
    need = randes.randes_rms_norm_backward_workspace(2000, 256)      # (few rows need none)
    big, bigs = torch.zeros(4, 2000, 256, device="cuda"), torch.ones(2000, device="cuda")
    many = dict(rows=2000, dy=big[0].data_ptr(), h=big[1].data_ptr(), dx=big[2].data_ptr(), rstd=bigs.data_ptr())
    ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    call = lambda at=ws.data_ptr(), n=ws.numel(), **kw: randes.randes_rms_norm_backward(randes.RmsNormBackward(**{**back, **kw}), at, n, s)
    cases = [(lambda: randes.rms_norm(x, gain[:100]), inv), (lambda: randes.rms_norm(x, gain.double()), inv), (lambda: randes.rms_norm(x, gain, x[:, :100]), inv),
             (lambda: randes.rms_norm(x, gain, x.bfloat16()), inv), (lambda: randes.rms_norm(x, gain, eps=0.0), inv), (lambda: randes.rms_norm(x, gain, eps=float("nan")), inv),
             (lambda: randes.rms_norm(torch.zeros(2, 32769, device="cuda")), inv), (lambda: randes.rms_norm(torch.zeros(2, 0, device="cuda")), inv),
             (lambda: randes.rms_norm(x, gain, h=f.h, y=f.h), inv), (lambda: randes.rms_norm(x, gain, x, packed=True, y=x), inv),
             (lambda: randes.rms_norm(x[1:], gain, h=x[:3]), inv), (lambda: randes.rms_norm(x.half(), gain), randes.UNSUPPORTED_DTYPE),
             (lambda: randes.rms_norm_backward(x, randes.pack8(x[:, :100]), f.rstd, gain), inv), (lambda: randes.rms_norm_backward(x, x, f.rstd[:2], gain), inv),
             (lambda: randes.rms_norm_backward(x, x.bfloat16(), f.rstd, gain), inv), (lambda: call(h=None), inv), (lambda: call(kept8=f.kept.address), inv),
             (lambda: call(rstd=None), inv), (lambda: call(dx=None), inv), (lambda: call(at=None, n=0, **many), randes.WORKSPACE_TOO_SMALL),
             (lambda: call(n=need - 1, **many), randes.WORKSPACE_TOO_SMALL), (lambda: call(at=ws.data_ptr() + 8, **many), randes.MISALIGNED),
             (lambda: call(dgain=gain.data_ptr() + 2), randes.MISALIGNED), (lambda: call(dtype=5), randes.UNSUPPORTED_DTYPE)]
    for i, (g, code) in enumerate(cases):
        with pytest.raises(randes.RandesError) as e:
            g()
        assert e.value.code == code, (i, e.value)
