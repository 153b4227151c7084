"""The differentiable token log probabilities, and packed weights, task-mixed products and token scores run together as a
serving program uses them."""
import subprocess
import sys
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2505_11204_b200 import build, randes, serve                    # noqa: E402
from paper_2505_11204_b200.scoring import token_log_probs                 # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def _reference(z, targets, scale):
    u = z.double() * scale
    lp = torch.log_softmax(u, 1)
    return lp.gather(1, targets.clamp(min=0)[:, None])[:, 0] * (targets >= 0), -(lp.exp() * lp).sum(1)


@pytest.mark.parametrize("use", ["both", "logprob", "entropy"])
def test_autograd_equals_the_fp64_graph(use):
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, vocab, scale = 9, 777, 0.75
    z = (torch.randn(n, vocab, generator=gen, device="cuda") * 2).requires_grad_(True)
    t = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    t[4] = -1                                              # a row that is not scored
    w = torch.randn(n, generator=gen, device="cuda")
    loss = lambda lp, h: (lp * w.to(lp.dtype)).sum() * (use != "entropy") + h.mean() * (use != "logprob")      # (an expanded gradient among them)
    lp, h = token_log_probs(z, t, scale)
    if use == "both":
        loss(lp, h).backward()
    else:
        ((lp * w).sum() if use == "logprob" else h.mean()).backward()
    zd = z.detach().double().requires_grad_(True)
    rlp, rh = _reference(zd, t, scale)
    loss(rlp, rh).backward()
    assert (lp.detach() - rlp).abs().max() < 2e-6 and (h.detach() - rh).abs().max() < 5e-6
    # both sides sum to zero over a row; elements are products of p with fp32 sums: a few units of 2^-20 of the largest
    assert (z.grad - zd.grad).abs().max() <= 2.0 ** -20 * (zd.grad.abs().max() + 1)


def test_autograd_without_gradients_and_with_strided_bf16_logits():
    z = torch.randn(6, 200, device="cuda").bfloat16()[:, :150].detach().requires_grad_(True)
    t = torch.arange(6, device="cuda")
    lp, h = token_log_probs(z, t)
    lp.sum().backward()                                    # the entropy's gradient never arrives
    assert z.grad.shape == z.shape and z.grad.dtype == torch.bfloat16 and torch.isfinite(z.grad).all()
    with torch.no_grad():
        a, b = token_log_probs(z, t)
    assert torch.equal(a, lp.detach()) and torch.equal(b, h.detach())


def test_serving_out_of_a_packed_superposition_agrees_with_the_retrieved_models():
    r = serve.serve(width=256, blocks=3, vocab=2003, n_tasks=3, n_tokens=7, steps=5)
    assert r["tokens"].shape == (5, 7) and ((r["tokens"] >= 0) & (r["tokens"] < 2003)).all()
    assert torch.isfinite(r["packed"]).all() and torch.isfinite(r["full"]).all()
    # four bits leave about a tenth of the weights' size as noise; the answers' log probabilities stay near
    assert (r["packed"] - r["full"]).abs().mean() < 0.5
    assert r["bytes"][0] > 6 * r["bytes"][1]
    wide = serve.serve(width=256, blocks=3, vocab=2003, n_tasks=3, n_tokens=21, steps=2)      # the form for more tokens
    assert torch.equal(wide["tokens"][0, :7], r["tokens"][0]) and (wide["packed"][0, :7] - r["packed"][0]).abs().max() < 1e-3


def test_a_new_task_learns_and_is_added():
    first, last, added = serve.learn()
    assert last > first + 1.0 and added


def test_the_command_runs():
    r = subprocess.run([sys.executable, "-m", "paper_2505_11204_b200.serve", "--width", "256", "--blocks", "2", "--vocab", "1001", "--steps", "3"],
                       cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "packed base and superposition" in r.stdout and "added to the superposition: yes" in r.stdout


def test_products_of_many_tokens_need_their_workspace():
    p = randes.pack(torch.randn(64, 256, device="cuda"))
    x, y = torch.randn(20, 256, device="cuda"), torch.empty(20, 64, device="cuda")
    need = randes.randes_packed_linear_workspace(64, 256, randes.F32, 20, False)
    assert need > 0 and randes.randes_packed_linear_workspace(64, 256, randes.F32, 8, True) == 0
    ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    call = lambda at, n: randes.randes_packed_linear(p.address, 64, 256, 64, x, 0, 256, 20, y, 0, 64, s, at, n)
    for at, n, code in ((None, 0, randes.WORKSPACE_TOO_SMALL), (ws.data_ptr(), need - 1, randes.WORKSPACE_TOO_SMALL),
                        (ws.data_ptr() + 8, need, randes.MISALIGNED)):
        with pytest.raises(randes.RandesError) as e:
            call(at, n)
        assert e.value.code == code
    call(ws.data_ptr(), need)
    assert torch.equal(y, randes.packed_linear(x, p))
