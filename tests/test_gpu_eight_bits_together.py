"""Eight-bit layers behind autograd, and the operators run together as serving and training programs use them."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2505_11204_b200 import build, randes, serve                    # noqa: E402
from paper_2505_11204_b200.training import norm_linear                    # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def eight(v):
    return randes.pack8(v).unpack().double()


def make(n, cols, rows, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, r = normal(n, cols).to(dtype), (3 * normal(n, cols)).to(dtype)
    gain, w = 1 + 0.2 * normal(cols), (normal(rows, cols) / cols ** 0.5).to(dtype)
    return x, r, gain, w, normal(n, rows).to(dtype), normal(n, cols).to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,cols,rows", [(1, 128, 40), (5, 200, 300), (300, 256, 513), (130, 1000, 64)])
def test_gradients_are_those_of_the_kept_values(n, cols, rows, dtype):
    x, r, gain, w, g, gh = make(n, cols, rows, dtype)
    leaves = [t.clone().requires_grad_(True) for t in (x, gain, w, r)]
    y, h = norm_linear(*leaves[:3], leaves[3])
    assert y.dtype is dtype and torch.equal(h.detach(), (x.float() + r.float()).to(dtype))
    torch.autograd.backward((y, h), (g, gh))
    half = torch.finfo(torch.bfloat16).eps / 2 if dtype is torch.bfloat16 else 0.0
    fp32 = 2.0 ** -18                                      # sums of up to a thousand exact products: far below this of the sum of magnitudes
    f = randes.rms_norm(x, gain, r, packed=True, checkpoint=True)
    n8, w8 = f.y.unpack().double(), eight(w)
    assert ((y.detach().double() - n8 @ w8.t()).abs() <= fp32 * (n8.abs() @ w8.abs().t()) + half * (n8 @ w8.t()).abs()).all()
    # the formulas of the module's documentation, in fp64, at the values that eight bits kept
    gr, gc = eight(g), eight(g.t().contiguous()).t()
    dw = gc.t() @ eight(f.y.unpack().t().contiguous()).t()
    size = gc.abs().t() @ n8.abs()
    assert ((leaves[2].grad.double() - dw).abs() <= fp32 * size + half * dw.abs()).all()
    wt = eight(w.t().contiguous())
    dn, dn_size = gr @ wt.t(), gr.abs() @ wt.abs().t()
    rs = f.rstd.double()[:, None]
    nd, gg, gs = f.kept.unpack().double() * rs, dn * gain.double(), dn_size * gain.double().abs()
    dx = rs * (gg - nd * (gg * nd).mean(1, keepdim=True)) + gh.double()
    off = fp32 * gs + half * gg.abs()                      # of every element of gg: its sum, and its rounding where it is stored in bf16
    tol = rs * (off + nd.abs() * (off * nd.abs()).mean(1, keepdim=True)) + fp32 * (rs * gs * (1 + nd.abs() * nd.abs().mean(1, keepdim=True)) + gh.double().abs()) + half * dx.abs()
    assert ((leaves[0].grad.double() - dx).abs() <= tol).all() and torch.equal(leaves[0].grad, leaves[3].grad)
    dgain = (dn * nd).sum(0)
    assert ((leaves[1].grad.double() - dgain).abs() <= ((fp32 * dn_size + half * dn.abs()) * nd.abs()).sum(0) + fp32 * (dn_size * nd.abs()).sum(0)).all()


def test_without_a_residual_without_a_gain_and_with_single_gradients():
    x, r, gain, w, g, gh = make(40, 300, 70, torch.float32)
    xs = x.clone().requires_grad_(True)
    y, h = norm_linear(xs, None, w)
    assert h is xs
    (y * g).sum().backward()
    ws = w.clone().requires_grad_(True)
    y2, _ = norm_linear(x, None, ws)
    assert torch.equal(y2, y)
    (y2 * g).sum().backward()
    both = [x.clone().requires_grad_(True), w.clone().requires_grad_(True)]
    (norm_linear(both[0], None, both[1])[0] * g).sum().backward()
    assert torch.equal(both[0].grad, xs.grad) and torch.equal(both[1].grad, ws.grad)
    rs = r.clone().requires_grad_(True)
    norm_linear(x, gain, w, rs)[1].sum().backward()        # only the residual stream: its gradient goes straight through (and arrives expanded)
    assert (rs.grad == 1).all()
    rs.grad = None
    norm_linear(x, gain, w, rs)[0].sum().backward()
    assert torch.isfinite(rs.grad).all()
    with torch.no_grad():
        assert torch.equal(norm_linear(x, gain, w, r)[0], norm_linear(x, gain, w, rs)[0].detach())


def test_a_layer_twice_and_shared_by_two_uses():
    x, r, gain, w, g, gh = make(30, 256, 256, torch.bfloat16)
    ws = w.clone().requires_grad_(True)
    y, h = norm_linear(x, gain, ws, r)
    y, h = norm_linear(y, gain, ws, h)
    (y.float().pow(2).mean() + h.float().pow(2).mean()).backward()
    assert torch.isfinite(ws.grad).all() and ws.grad.dtype is torch.bfloat16 and ws.grad.abs().sum() > 0


def test_a_step_is_captured_and_replayed():
    x, r, gain, w, g, gh = make(200, 512, 256, torch.bfloat16)
    for _ in range(2):
        f = randes.rms_norm(x, gain, r, packed=True, checkpoint=True)
        wp, wt = randes.pack8_both(w)
    torch.cuda.synchronize()

    def step():
        f = randes.rms_norm(x, gain, r, packed=True, checkpoint=True)
        p, pt = randes.pack8_both(w)
        y = randes.packed8_linear(f.y, p, y_dtype=randes.BF16)
        q, qt = randes.pack8_both(g)
        dw = randes.packed8_linear(qt, randes.pack8_transposed(f.y))
        dx, dgain = randes.rms_norm_backward(randes.packed8_linear(q, pt, y_dtype=randes.BF16), f.kept, f.rstd, gain, dh=gh)
        return y, dw, dx, dgain

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (1, 2):
        for to, new in zip((x, r, gain, w, g, gh), make(200, 512, 256, torch.bfloat16, seed)):
            to.copy_(new)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))


def test_autograd_is_captured_and_replayed():
    made = make(200, 512, 256, torch.bfloat16)
    x, r, gain, w, g, gh = [t.clone() for t in made]
    leaves = [t.requires_grad_(True) for t in (x, gain, w, r)]

    def step():
        y, h = norm_linear(x, gain, w, r)
        return torch.autograd.grad([y, h], leaves, [g, gh])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (1, 2):
        with torch.no_grad():
            for to, new in zip((x, r, gain, w, g, gh), make(200, 512, 256, torch.bfloat16, seed)):
                to.copy_(new)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))


def test_two_threads_with_streams_of_their_own():
    import threading

    made = [make(150 + 100 * i, 512 + 256 * i, 256, torch.bfloat16, i) for i in range(2)]

    def step(x, r, gain, w, g, gh):
        f = randes.rms_norm(x, gain, r, packed=True, checkpoint=True)
        p, pt = randes.pack8_both(w)
        q, qt = randes.pack8_both(g)
        dx, dgain = randes.rms_norm_backward(randes.packed8_linear(q, pt, y_dtype=randes.BF16), f.kept, f.rstd, gain, dh=gh)
        return randes.packed8_linear(f.y, p), randes.packed8_linear(x[:7], p), randes.packed8_linear(qt, randes.pack8_transposed(f.y)), dx, dgain

    want, wrong = [step(*m) for m in made], []
    torch.cuda.synchronize()

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got = step(*made[i])
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_prompts_in_eight_bits_agree_with_the_retrieved_models():
    r = serve.read_prompts(width=256, blocks=3, vocab=2003, n_tasks=3, n_tokens=131)
    assert torch.isfinite(r["eight"]).all() and r["eight"].shape == (3, 130)
    # eight bits leave about 2^-5 of a product's size as noise, the logits have unit size
    assert (r["eight"] - r["full"]).abs().mean() < 0.2
    assert r["bytes"][0] > 2 * r["bytes"][1]


def test_tuning_a_layer_runs():
    first, last, added = serve.tune()
    assert first == first and last == last and added


def test_the_command_reads_prompts():
    r = subprocess.run([sys.executable, "-m", "paper_2505_11204_b200.serve", "--width", "256", "--blocks", "2", "--vocab", "1001", "--steps", "2", "--prompt", "70"],
                       cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "prompts of 70 tokens" in r.stdout and "added: yes" in r.stdout
