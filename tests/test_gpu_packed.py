"""Four-bit weights on the GPU: what pack writes and unpack reads back, the retrieved weight packed directly, and the
products of a few tokens with packed matrices, against plain numpy implementations of the definitions.

* Packing is a function of exactly rounded steps (two fp32 quotients, one bf16 rounding, one rounding to an integer), so
  the values read back must equal the numpy ones bit for bit.
* Dyadic inputs to the products (weights whose scales are powers of two, activations on a grid of 1/16): every partial
  sum is exact in fp32 in any order, so the result must equal the fp64 definition bit for bit.  A wrong nibble, scale,
  sign, slot or token fails this.
* Gaussian inputs: products are exact, sums run in fp32.  As for the dense linear layer the accepted error is the
  random-walk form sqrt(2 n + 2) * 2^-24 * y_abs, n the number of products of one output and y_abs the sum of their
  magnitudes: n roundings of 2^-24 of partial sums that stay near y_abs / sqrt(n)."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import randes_oracle as ro                              # noqa: E402
from paper_2505_11204_b200 import build, randes, workloads as wl    # noqa: E402
from gpu_util import model_to_dev, to_dev                           # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
S, F = wl.SHUFFLE, wl.FLIP
TYPES = {wl.F32: torch.float32, wl.BF16: torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build_library()


def bf16_round(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).bfloat16().float().numpy()


def packed_values(w, group):
    """The definition, on an fp32 array [rows, cols]: the values that four bits keep."""
    rows, cols = w.shape
    out = np.empty_like(w)
    with np.errstate(all="ignore"):
        for c0 in range(0, cols, group):
            p = w[:, c0:c0 + group]
            a = np.abs(p).max(axis=1)
            s = bf16_round(a / np.float32(7))
            s = np.where(s >= np.float32(2.0 ** -100), s, np.float32(0))
            q = np.where(s[:, None] > 0, np.clip(np.rint(p / np.where(s > 0, s, 1)[:, None]), -7, 7), 0)
            v = q.astype(np.float32) * s[:, None]
            v[~np.isfinite(p).all(axis=1)] = np.nan
            out[:, c0:c0 + group] = v
    return out


def same_values(got, want, what=""):
    got, want = np.asarray(got, dtype=np.float32), np.asarray(want, dtype=np.float32)
    assert np.array_equal(got, want, equal_nan=True), "%s: %d of %d values differ" % (what, int((~((got == want) | (np.isnan(got) & np.isnan(want)))).sum()), got.size)


def weight(rng, rows, cols, dtype):
    w = (rng.standard_normal((rows, cols)) * 0.02).astype(np.float32)
    return bf16_round(w) if dtype == wl.BF16 else w


def on_gpu(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(TYPES[dtype])


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 64), (16, 128), (17, 65), (5, 31), (33, 200), (100, 1000), (257, 513), (3, 4097)])
def test_pack_and_unpack_equal_the_definition(rows, cols, group, dtype):
    w = weight(np.random.default_rng(rows * 7919 + cols), rows, cols, dtype)
    p = randes.pack(on_gpu(w, dtype), group=group)
    assert p.nbytes == randes.randes_packed_bytes(rows, cols, group)
    want = packed_values(w, group)
    same_values(p.unpack().cpu().numpy(), want, "fp32")
    same_values(p.unpack(out_dtype=wl.BF16).float().cpu().numpy(), bf16_round(want), "bf16")


def test_quotients_next_to_ties_round_as_the_definition():
    # weights that sit on, just above and just below half a step of their group's scale, over many scales
    rng = np.random.default_rng(3)
    rows, cols = 64, 256
    w = np.zeros((rows, cols), dtype=np.float32)
    for r in range(rows):
        for c0 in range(0, cols, 32):
            top = np.float32(2.0 ** rng.uniform(-90, 90))
            s = bf16_round(np.array([top / np.float32(7)]))[0]
            k = rng.integers(-7, 7, size=32) + 0.5
            v = (k * np.float64(s)).astype(np.float32)
            v = np.nextafter(v, np.float32(np.inf) * rng.choice([-1, 1], size=32)) if r % 3 == 1 else v
            w[r, c0:c0 + 32] = np.clip(v, -top, top)
            w[r, c0] = top
    got = randes.pack(on_gpu(w, wl.F32), group=32).unpack().cpu().numpy()
    same_values(got, packed_values(w, 32))


def test_zero_tiny_huge_and_non_finite_groups():
    w = np.zeros((20, 256), dtype=np.float32)
    rng = np.random.default_rng(4)
    w[1] = rng.standard_normal(256)
    w[2, :] = 1e-38
    w[3, :] = 1e-45
    w[4, :] = np.float32(2.0 ** -97)                     # scale 2^-97 / 7 = 2^-99.8: just kept
    w[11, :] = np.float32(2.0 ** -98)                    # scale 2^-100.8: below the smallest kept
    w[5, :] = np.float32(7 * 2.0 ** -100)                # exactly the smallest kept
    w[6, 3], w[6, 4] = np.finfo(np.float32).max, -1.0
    w[7], w[7, 70] = rng.standard_normal(256), np.nan
    w[8], w[8, 200] = rng.standard_normal(256), np.inf
    w[9], w[9, 0] = rng.standard_normal(256), -np.inf
    w[10, 64:128] = -0.0
    for group in (32, 64, 128):
        want = packed_values(w, group)
        same_values(randes.pack(on_gpu(w, wl.F32), group=group).unpack().cpu().numpy(), want, "group %d" % group)
        assert np.isnan(want[7]).sum() == group and np.isnan(want[8]).sum() == group and not np.isnan(want[6]).any()
        assert want[4].all() and want[5].all() and not want[11].any()


def test_strided_and_misaligned_weights_and_lists():
    rng = np.random.default_rng(5)
    shapes = [(40, 96), (7, 64), (1, 500), (18, 129), (0, 64), (5, 0)] + [(16 + i, 32 + i) for i in range(40)]
    for dtype in (wl.F32, wl.BF16):
        tensors, arrays = [], []
        for i, (r, c) in enumerate(shapes):
            w = weight(rng, r, c, dtype)
            off, pad = i % 3, 8 * (i % 2) + i % 5
            store = torch.full((off + r * (c + pad) + 8,), float("nan"), device="cuda", dtype=TYPES[dtype])
            t = store[off:off + r * (c + pad)].view(r, c + pad)[:, :c]
            t.copy_(on_gpu(w, dtype))
            tensors.append(t)
            arrays.append(w)
        before = randes.randes_launch_count()
        packed = randes.pack(tensors, group=64)
        assert randes.randes_launch_count() - before == 2          # 44 matrices that hold anything, 32 per launch
        for p, w in zip(packed, arrays):
            same_values(p.unpack().cpu().numpy(), packed_values(w, 64), str(w.shape))
        # strided output
        wide = torch.full((40, 200), -1.0, device="cuda")
        packed[0].unpack(out=wide[:, 3:99])
        same_values(wide[:, 3:99].cpu().numpy(), packed_values(arrays[0], 64))
        assert (wide[:, :3] == -1).all() and (wide[:, 99:] == -1).all()


def _plan(rows, cols, members, flags, storage, m_dtype, ids=(3, 0, 8), seeds=(42, 43, 2 ** 35 + 1), extra=()):
    """A plan of `members` same-shape layers (one group) and single layers `extra`."""
    r, c, g, fl = [rows] * members, [cols] * members, [0] * members, [flags]
    for k, (er, ec) in enumerate(extra):
        r.append(er); c.append(ec); g.append(k + 1); fl.append(F)
    spec = (r, c, g, fl)
    return randes.Plan(r, c, g, fl, storage=storage, m_dtype=m_dtype, task_ids=ids, seeds=seeds), spec, list(ids), list(seeds)


@pytest.mark.parametrize("storage,m_dtype", [(wl.F32, wl.F32), (wl.BF16, wl.BF16), (wl.BF16, wl.F32), (wl.F32, wl.BF16)])
def test_retrieve_packed_packs_what_retrieve_returns(storage, m_dtype):
    for rows, cols, flags in ((40, 264, S | F), (17, 130, F), (33, 64, S), (8, 1000, S | F)):
        plan, _, ids, _ = _plan(rows, cols, 4, flags, storage, m_dtype, extra=[(5, 77)])
        rng = np.random.default_rng(rows)
        base = [on_gpu(weight(rng, r, c, storage), storage) for r, c in zip(plan.rows, plan.cols)]
        M = plan.new_superposition()
        for l in range(plan.n_layers):
            plan.slot(M, l).copy_(torch.randn(plan.rows[l], plan.cols[l], device="cuda") * 3e-3)
        for t in ids:
            want = plan.retrieve(t, 0.37, base, M)
            for group in (32, 128):
                got = plan.retrieve_packed(t, 0.37, base, M, group=group)
                for l in range(plan.n_layers):
                    same_values(got[l].unpack().cpu().numpy(), packed_values(want[l].cpu().numpy(), group), "task %d layer %d" % (t, l))
        some = plan.retrieve_packed(ids[1], 0.37, base, M, group=64, layers=[4, 1])
        assert [(p.rows, p.cols) for p in some] == [(5, 77), (rows, cols)]
        same_values(some[1].unpack().cpu().numpy(), packed_values(plan.retrieve(ids[1], 0.37, base, M)[1].cpu().numpy(), 64))
        plan.close()


def test_pack_superposition_packs_every_slot():
    plan, _, _, _ = _plan(24, 96, 3, S | F, wl.BF16, wl.F32, extra=[(9, 40)])
    M = plan.new_superposition()
    M.normal_()
    for l, p in enumerate(plan.pack_superposition(M, group=32)):
        same_values(p.unpack().cpu().numpy(), packed_values(plan.slot(M, l).cpu().numpy(), 32))
    some = plan.pack_superposition(M, slots=[2])
    assert some[0] is None and some[2].rows == 24 and len(some) == 4
    plan.close()


def dyadic_weight(rng, rows, cols, group):
    """Values q * 2^-k with a 7 in every group: the scale is the power of two itself."""
    w = np.zeros((rows, cols), dtype=np.float32)
    for c0 in range(0, cols, group):
        n = min(group, cols - c0)
        s = np.float32(2.0) ** -rng.integers(4, 8, size=(rows, 1)).astype(np.float32)
        q = rng.integers(-7, 8, size=(rows, n))
        q[np.arange(rows), rng.integers(0, n, size=rows)] = 7
        w[:, c0:c0 + n] = q * s
    return w


def dyadic_acts(rng, n, cols):
    return (rng.integers(-8, 9, size=(n, cols)) / 16.0).astype(np.float32)


@pytest.mark.parametrize("x_dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 64), (15, 63), (50, 65), (100, 200), (300, 768), (33, 1032), (20, 4100), (3000, 64)])
def test_linear_is_exact_on_dyadic_inputs(rows, cols, group, x_dtype):
    rng = np.random.default_rng(rows + cols)
    w = dyadic_weight(rng, rows, cols, group)
    p = randes.pack(on_gpu(w, wl.F32), group=group)
    for n in (1, 2, 8, 9, 17, 40, 64, 65, 131):
        x = dyadic_acts(rng, n, cols)
        want = x.astype(np.float64) @ w.astype(np.float64).T
        y = torch.full((n, rows), float("nan"), device="cuda")
        assert randes.packed_linear(on_gpu(x, x_dtype), p, y=y) is y
        same_values(y.cpu().numpy(), want, "%d tokens" % n)
        same_values(randes.packed_linear(on_gpu(x, x_dtype), p, y_dtype=wl.BF16).float().cpu().numpy(), bf16_round(want), "%d tokens, bf16" % n)


def test_linear_strided_and_misaligned_tensors_leave_the_rest_alone():
    rng = np.random.default_rng(6)
    rows, cols, n = 70, 136, 11
    w = dyadic_weight(rng, rows, cols, 64)
    p = randes.pack(on_gpu(w, wl.F32), group=64)
    x = dyadic_acts(rng, n, cols)
    want = x.astype(np.float64) @ w.astype(np.float64).T
    for dtype in (wl.F32, wl.BF16):
        for off, pad in ((0, 8), (0, 3), (1, 0), (3, 5), (8, 16)):
            store = torch.full((off + n * (cols + pad),), float("nan"), device="cuda", dtype=TYPES[dtype])
            xt = store[off:].view(n, cols + pad)[:, :cols]
            xt.copy_(on_gpu(x, dtype))
            out = torch.full((n, rows + 9), -5.0, device="cuda", dtype=TYPES[dtype])
            randes.packed_linear(xt, p, y=out[:, 4:4 + rows])
            got = out[:, 4:4 + rows].float().cpu().numpy()
            same_values(got, bf16_round(want) if dtype == wl.BF16 else want, "offset %d pad %d" % (off, pad))
            assert (out[:, :4] == -5).all() and (out[:, 4 + rows:] == -5).all()


@pytest.mark.parametrize("x_dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("rows,cols,group", [(768, 768, 64), (513, 2049, 32), (64, 8192, 128), (5000, 130, 64)])
def test_linear_on_gaussian_inputs(rows, cols, group, x_dtype):
    rng = np.random.default_rng(cols)
    p = randes.pack(on_gpu(weight(rng, rows, cols, wl.F32), wl.F32), group=group)
    w = p.unpack().cpu().numpy().astype(np.float64)
    for n in (1, 7, 33):
        x = rng.standard_normal((n, cols)).astype(np.float32)
        x = bf16_round(x) if x_dtype == wl.BF16 else x
        y = randes.packed_linear(on_gpu(x, x_dtype), p)
        want, y_abs = x.astype(np.float64) @ w.T, np.abs(x.astype(np.float64)) @ np.abs(w).T
        err = np.abs(y.cpu().numpy().astype(np.float64) - want)
        tol = np.sqrt(2.0 * cols + 2.0) * 2.0 ** -24 * y_abs
        assert (err <= tol).all(), "worst %.3g x tolerance" % float((err / tol).max())
        assert torch.equal(randes.packed_linear(on_gpu(x, x_dtype), p, y_dtype=wl.BF16), y.bfloat16())
        assert torch.equal(randes.packed_linear(on_gpu(x, x_dtype), p), y)      # the same bits every time


@pytest.mark.parametrize("group", [32, 64, 128])
def test_few_tokens_on_a_large_matrix(group):
    """Sizes on either side of where fp32 activations change over to the other form; a superposition counts as well."""
    rng = np.random.default_rng(12)
    for rows, cols in ((8192, 4096), (8191, 4096), (4100, 8193)):
        p = randes.pack(on_gpu(weight(rng, rows, cols, wl.F32), wl.F32), group=group)
        w = p.unpack().double()
        for n in (1, 3, 8):
            x = rng.standard_normal((n, cols)).astype(np.float32)
            for dtype in (wl.F32, wl.BF16):
                xt = on_gpu(x, dtype)
                y = randes.packed_linear(xt, p)
                want, y_abs = xt.double() @ w.T, xt.double().abs() @ w.abs().T
                assert ((y.double() - want).abs() <= np.sqrt(2.0 * cols + 2.0) * 2.0 ** -24 * y_abs).all(), (rows, cols, n, dtype)


def test_linear_with_extreme_activations():
    rng = np.random.default_rng(8)
    rows, cols = 32, 128
    w = dyadic_weight(rng, rows, cols, 64)
    w[w == 0] = np.float32(2.0 ** -7)                      # no zero code: an infinity times zero would be a NaN
    p = randes.pack(on_gpu(w, wl.F32), group=64)
    v = p.unpack().cpu().numpy().astype(np.float64)
    assert (v != 0).sum() > 0
    x = np.zeros((6, cols), dtype=np.float32)
    x[0, 5] = 3e38                                         # above the largest finite bf16 when rounded, not when truncated
    x[1, 9] = 1e-30
    x[2, 7] = np.float32(1) + np.float32(2.0 ** -23)       # needs all 24 bits
    x[3] = rng.standard_normal(cols)
    x[4, 3] = np.inf
    x[5, 3] = np.nan
    y = randes.packed_linear(on_gpu(x, wl.F32), p).cpu().numpy()
    with np.errstate(all="ignore"):
        for b in range(3):
            # 24 + 3 bits do not fit fp32: the accepted error of this file (a single product errs by far less)
            want, y_abs = x[b].astype(np.float64) @ v.T, np.abs(x[b].astype(np.float64)) @ np.abs(v).T
            assert (np.abs(y[b] - want) <= np.sqrt(2.0 * cols + 2.0) * 2.0 ** -24 * y_abs).all(), b
    live = v[:, 3] != 0
    assert np.array_equal(y[4][live], np.sign(v[live, 3]) * np.inf) and np.isnan(y[4][~live]).all()
    assert np.isnan(y[5]).all()
    # tokens do not see one another: the ordinary one next to them is what it is alone
    assert np.array_equal(y[3], randes.packed_linear(on_gpu(x[3:4], wl.F32), p).cpu().numpy()[0])


def test_linear_reads_back_a_group_with_a_nan_as_nan():
    rng = np.random.default_rng(9)
    w = weight(rng, 40, 256, wl.F32)
    w[21, 100] = np.nan
    y = randes.packed_linear(on_gpu(rng.standard_normal((3, 256)), wl.BF16), randes.pack(on_gpu(w, wl.F32), group=64)).cpu().numpy()
    assert np.isnan(y[:, 21]).all() and np.isfinite(np.delete(y, 21, axis=1)).all()


def _signs(spec, seed, task, slot, cols):
    flagged = spec[3][spec[2][slot]] & F
    return ro.sign_row(seed, task, slot, cols).astype(np.float64) if flagged else np.ones(cols)


def _tasks_reference(spec, ids, seeds, task_ids, lam, layer, x, base, m):
    """fp64 definition and the sum of magnitudes; base, m: the packed values."""
    seed = dict(zip(ids, seeds))
    x = x.astype(np.float64)
    y, y_abs = x @ base.T, np.abs(x) @ np.abs(base).T
    for b, t in enumerate(task_ids):
        slot = int(ro.task_tables(spec, seed[t], t)[1][layer])
        xs = x[b] * _signs(spec, seed[t], t, slot, x.shape[1])
        y[b] += lam * (m[slot] @ xs)
        y_abs[b] += abs(lam) * (np.abs(m[slot]) @ np.abs(xs))
    return y, y_abs


@pytest.mark.parametrize("x_dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("flags", [S | F, S, F, 0])
@pytest.mark.parametrize("rows,cols,group", [(16, 64, 64), (50, 130, 32), (31, 1100, 128), (600, 200, 64)])
def test_tasks_are_exact_on_dyadic_inputs(rows, cols, group, flags, x_dtype):
    plan, spec, ids, seeds = _plan(rows, cols, 5, flags, wl.BF16, wl.BF16, ids=[3, 0, 8, 77], seeds=[42, 43, 2 ** 35 + 1, 9])
    rng = np.random.default_rng(rows)
    base = dyadic_weight(rng, rows, cols, group)
    m = [dyadic_weight(rng, rows, cols, group) for _ in range(5)]
    pb, pm = randes.pack(on_gpu(base, wl.F32), group=group), randes.pack([on_gpu(v, wl.F32) for v in m], group=group)
    lam = 0.25
    for n in (1, 3, 8, 20, 64, 100):
        x = dyadic_acts(rng, n, cols)
        tasks = [ids[int(k)] for k in rng.integers(0, len(ids), size=n)]
        for layer in (0, 3):
            want, _ = _tasks_reference(spec, ids, seeds, tasks, lam, layer, x, base.astype(np.float64), [v.astype(np.float64) for v in m])
            y = torch.full((n, rows), float("nan"), device="cuda")
            plan.packed_linear(tasks, lam, layer, on_gpu(x, x_dtype), pb, pm, y=y)
            same_values(y.cpu().numpy(), want, "%d tokens, layer %d" % (n, layer))
    plan.close()


def test_tasks_with_many_slots_and_unused_slots_missing():
    ids, seeds = list(range(40)), [100 + i for i in range(40)]
    rows, cols, members = 48, 320, 24
    plan, spec, ids, seeds = _plan(rows, cols, members, S | F, wl.BF16, wl.BF16, ids=ids, seeds=seeds)
    rng = np.random.default_rng(12)
    base = dyadic_weight(rng, rows, cols, 64)
    m = [dyadic_weight(rng, rows, cols, 64) for _ in range(members)]
    tasks = [ids[int(k)] for k in rng.integers(0, 40, size=64)]
    used = {int(ro.task_tables(spec, seeds[t], t)[1][2]) for t in tasks}
    assert len(used) > 10
    pm = [randes.pack(on_gpu(v, wl.F32)) if l in used else None for l, v in enumerate(m)]
    x = dyadic_acts(rng, 64, cols)
    want, _ = _tasks_reference(spec, ids, seeds, tasks, 0.5, 2, x, base.astype(np.float64), [v.astype(np.float64) for v in m])
    same_values(plan.packed_linear(tasks, 0.5, 2, on_gpu(x, wl.BF16), randes.pack(on_gpu(base, wl.F32)), pm).cpu().numpy(), want)
    # a slot with a NaN reaches the tokens of the tasks that keep the layer there, and no others
    slot = int(ro.task_tables(spec, seeds[tasks[5]], tasks[5])[1][2])
    bad = m[slot].copy()
    bad[7, 3] = np.nan
    pm[slot] = randes.pack(on_gpu(bad, wl.F32))
    y = plan.packed_linear(tasks, 0.5, 2, on_gpu(x, wl.BF16), randes.pack(on_gpu(base, wl.F32)), pm).cpu().numpy()
    hit = np.array([int(ro.task_tables(spec, seeds[t], t)[1][2]) == slot for t in tasks])
    assert np.isnan(y[hit, 7]).all() and hit.any()
    same_values(np.delete(y, 7, axis=1), np.delete(want, 7, axis=1))
    same_values(y[~hit], want[~hit])
    plan.close()


@pytest.mark.parametrize("x_dtype", [wl.F32, wl.BF16])
def test_tasks_on_gaussian_inputs(x_dtype):
    rows, cols = 300, 1536
    plan, spec, ids, seeds = _plan(rows, cols, 4, S | F, wl.BF16, wl.BF16)
    rng = np.random.default_rng(13)
    pb = randes.pack(on_gpu(weight(rng, rows, cols, wl.F32), wl.F32))
    pm = randes.pack([on_gpu(weight(rng, rows, cols, wl.F32), wl.F32) for _ in range(4)])
    vb, vm = pb.unpack().cpu().numpy().astype(np.float64), [p.unpack().cpu().numpy().astype(np.float64) for p in pm]
    for n in (1, 5, 30):
        x = rng.standard_normal((n, cols)).astype(np.float32)
        x = bf16_round(x) if x_dtype == wl.BF16 else x
        tasks = [ids[b % 3] for b in range(n)]
        y = plan.packed_linear(tasks, 0.3, 1, on_gpu(x, x_dtype), pb, pm)
        want, y_abs = _tasks_reference(spec, ids, seeds, tasks, float(np.float32(0.3)), 1, x, vb, vm)
        err, tol = np.abs(y.cpu().numpy().astype(np.float64) - want), np.sqrt(4.0 * cols + 2.0) * 2.0 ** -24 * y_abs
        assert (err <= tol).all(), "worst %.3g x tolerance" % float((err / tol).max())
    plan.close()


def test_empty_calls_and_columns():
    p = randes.pack(torch.zeros(32, 64, device="cuda"))
    assert randes.packed_linear(torch.zeros(0, 64, device="cuda"), p).shape == (0, 32)
    empty = randes.pack(torch.zeros(8, 0, device="cuda"))
    y = torch.full((3, 8), 7.0, device="cuda")
    randes.packed_linear(torch.zeros(3, 0, device="cuda"), empty, y=y)
    assert (y == 0).all()                                  # a sum over no columns
    assert randes.packed_linear(torch.zeros(3, 64, device="cuda"), randes.pack(torch.zeros(0, 64, device="cuda"))).shape == (3, 0)
    assert randes.pack([]) == []


def _refused(code, fn):
    with pytest.raises(randes.RandesError) as e:
        fn()
    assert e.value.code == code, (e.value.code, str(e.value))


def test_refusals():
    inv, mis, dt = randes.INVALID_ARGUMENT, randes.MISALIGNED, randes.UNSUPPORTED_DTYPE
    w = torch.randn(32, 128, device="cuda")
    p = randes.pack(w)
    x = torch.randn(4, 128, device="cuda")
    before = randes.randes_launch_count()
    _refused(inv, lambda: randes.pack(w, group=48))
    _refused(dt, lambda: randes.pack(w.half()))
    _refused(inv, lambda: randes.pack(w.t()))
    _refused(inv, lambda: randes.pack([w, w.bfloat16()]))
    _refused(inv, lambda: randes.pack(w[0]))
    _refused(inv, lambda: randes.pack(w[:1].expand(32, 128)))
    _refused(inv, lambda: p.unpack(out=torch.empty(32, 127, device="cuda")))
    _refused(inv, lambda: randes.packed_linear(x[:, :64], p))
    _refused(dt, lambda: randes.packed_linear(x.double(), p))
    _refused(inv, lambda: randes.packed_linear(x, p, y=torch.empty(4, 31, device="cuda")))
    _refused(inv, lambda: randes.packed_linear(x.cpu(), p))
    s = torch.cuda.current_stream().cuda_stream
    y = torch.empty(4, 32, device="cuda")
    call = lambda packed=p.address, rows=32, cols=128, group=64, xp=x.data_ptr(), xd=0, xs=128, n=4, yp=y.data_ptr(), yd=0, ys=32: \
        randes.randes_packed_linear(packed, rows, cols, group, xp, xd, xs, n, yp, yd, ys, s)
    _refused(inv, lambda: call(packed=None))
    _refused(mis, lambda: call(packed=p.address + 8))
    _refused(inv, lambda: call(group=16))
    _refused(dt, lambda: call(xd=5))
    _refused(dt, lambda: call(yd=-1))
    _refused(mis, lambda: call(xp=x.data_ptr() + 2))
    _refused(mis, lambda: call(yp=y.data_ptr() + 1))
    _refused(inv, lambda: call(xs=127))
    _refused(inv, lambda: call(ys=31))
    _refused(inv, lambda: call(yp=x.data_ptr()))
    _refused(inv, lambda: call(yp=p.address))
    _refused(inv, lambda: call(xp=None))
    _refused(inv, lambda: call(rows=70000, cols=70000, xs=70000, ys=70000))
    mat = (randes.Matrix * 1)(randes.Matrix(w.data_ptr(), 32, 128, 128))
    _refused(inv, lambda: randes.randes_pack(mat, 1, 0, 64, (ctypes.c_void_p * 1)(None), s))
    _refused(mis, lambda: randes.randes_pack(mat, 1, 0, 64, (ctypes.c_void_p * 1)(p.address + 4), s))
    _refused(inv, lambda: randes.randes_pack(mat, 1, 0, 64, (ctypes.c_void_p * 1)(w.data_ptr()), s))
    _refused(inv, lambda: randes.randes_pack(None, 1, 0, 64, None, s))
    assert randes.randes_packed_bytes(32, 128, 40) == 0 and randes.randes_packed_bytes(0, 128, 32) == 0
    plan, _, ids, _ = _plan(32, 128, 3, S | F, wl.F32, wl.F32)
    M = plan.new_superposition().zero_()
    base = [w, w, w]
    pm = plan.pack_superposition(M)
    _refused(randes.UNKNOWN_TASK, lambda: plan.retrieve_packed(99, 1.0, base, M))
    _refused(inv, lambda: plan.retrieve_packed(ids[0], 1.0, base, M, layers=[3]))
    _refused(randes.UNKNOWN_TASK, lambda: plan.packed_linear([ids[0], 99, 0, 0], 1.0, 0, x, p, pm))
    _refused(inv, lambda: plan.packed_linear(ids[:1], 1.0, 0, x, p, pm))
    _refused(inv, lambda: plan.packed_linear([ids[0]] * 4, 1.0, 0, x, p, [None] * 3))
    _refused(inv, lambda: plan.packed_linear([ids[0]] * 4, 1.0, 0, x, p, pm[:2]))
    _refused(inv, lambda: plan.packed_linear([ids[0]] * 4, 1.0, 0, x, p, plan.pack_superposition(M, group=32)))
    _refused(inv, lambda: plan.packed_linear([ids[0]] * 4, 1.0, 0, x, randes.pack(w[:16]), pm))
    gauss = randes.Plan([32], [128], [0], [randes.GAUSS], task_ids=[0], seeds=[1])
    _refused(inv, lambda: gauss.retrieve_packed(0, 1.0, [w], gauss.new_superposition()))
    _refused(inv, lambda: gauss.packed_linear([0] * 4, 1.0, 0, x, p, [p]))
    lone = randes.randes_launch_count() - before
    assert lone == 4                                       # the five packs that were meant to work: two of them in one launch each
    gauss.close()
    plan.close()


def test_side_stream_and_graph_replay():
    rng = np.random.default_rng(14)
    w = dyadic_weight(rng, 64, 256, 64)
    p = randes.pack(on_gpu(w, wl.F32))
    x = on_gpu(dyadic_acts(rng, 3, 256), wl.BF16)
    y = torch.empty(3, 64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        randes.packed_linear(x, p, y=y)
    side.synchronize()
    want = x.double().cpu().numpy() @ w.astype(np.float64).T
    same_values(y.cpu().numpy(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        randes.packed_linear(x, p, y=y)
    for _ in range(2):
        new = dyadic_acts(rng, 3, 256)
        x.copy_(on_gpu(new, wl.BF16))
        graph.replay()
        torch.cuda.synchronize()
        same_values(y.cpu().numpy(), new.astype(np.float64) @ w.astype(np.float64).T)


_TWO_THREADS = """
import sys, threading
sys.path.insert(0, {root!r})
import torch
from paper_2505_11204_b200 import randes
torch.cuda.init()
torch.manual_seed({seed})
failed = []
for dtype in (torch.float32, torch.bfloat16):
    for group in (32, 64, 128):
        # more rows, fewer CTAs to a row block: every size wants another amount of shared memory
        packed = [randes.pack(torch.randn(rows, 1024, device="cuda"), group=group) for rows in (64, 2048, 16384, 40000)]
        xs = [torch.randn(n, 1024, device="cuda").to(dtype) for n in range(1, 9)]
        torch.cuda.synchronize()
        for p in packed:
            start = threading.Barrier(len(xs))

            def work(x):
                try:
                    torch.cuda.current_stream()
                    start.wait()
                    for _ in range(3):
                        randes.packed_linear(x, p)
                except Exception as e:
                    failed.append((str(dtype), group, p.rows, x.shape[0], str(e)))

            threads = [threading.Thread(target=work, args=(x,)) for x in xs]
            for t in threads: t.start()
            for t in threads: t.join()
            for x in xs[::-1]:
                try:
                    y = randes.packed_linear(x, p)
                    assert torch.equal(y, randes.packed_linear(x, p))
                except Exception as e:
                    failed.append(("after", str(dtype), group, p.rows, x.shape[0], str(e)))
torch.cuda.synchronize()
print(len(failed), failed[:3])
sys.exit(1 if failed else 0)
"""


def test_first_calls_from_several_threads_at_once():
    """Threads whose calls want different amounts of shared memory, each kernel's first calls among them (so in processes of
    their own)."""
    for seed in range(4):
        r = subprocess.run([sys.executable, "-c", _TWO_THREADS.format(root=ROOT, seed=seed)], cwd=ROOT, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, (seed, r.stdout[-2000:], r.stderr[-2000:])


@pytest.mark.parametrize("rows,cols", [(4096, 4096), (4096, 4095), (16384, 1024)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_few_tokens_on_a_large_superposition(rows, cols, group):
    """Sizes on either side of where fp32 activations change over to the other form, the superposition's columns counted; the
    workspace is of the size that is asked for and no larger."""
    plan, spec, ids, seeds = _plan(rows, cols, 5, S | F, wl.BF16, wl.BF16, ids=[3, 0, 8, 77], seeds=[42, 43, 2 ** 35 + 1, 9])
    rng = np.random.default_rng(21)
    pb = randes.pack(on_gpu(weight(rng, rows, cols, wl.F32), wl.F32), group=group)
    pm = randes.pack([torch.randn(rows, cols, device="cuda") * 3e-3 for _ in range(5)], group=group)
    base, m = pb.unpack().double(), [p.unpack().double() for p in pm]
    lam = float(np.float32(0.3))
    for n in (1, 3, 8):
        tasks = [ids[(3 * b + 1) % 4] for b in range(n)]
        slots = [int(ro.task_tables(spec, seeds[ids.index(t)], t)[1][2]) for t in tasks]
        assert n < 3 or len(set(slots)) > 1
        x = torch.randn(n, cols, device="cuda")
        need = randes.randes_packed_linear_workspace(rows, cols, wl.F32, n, True)
        assert (need > 0) == ((rows, cols) != (4096, 4095))
        ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        y = torch.full((n, rows), float("nan"), device="cuda")
        addresses = (ctypes.c_void_p * 5)(*[p.address for p in pm])
        randes.randes_packed_linear_tasks(plan.handle, 0.3, 2, group, (ctypes.c_uint32 * n)(*tasks), n, x, 0, cols, pb.address, addresses, y, 0, rows,
                                          torch.cuda.current_stream().cuda_stream, ws, need)
        assert (ws[need:] == 0xA5).all()
        assert torch.equal(y, plan.packed_linear(tasks, 0.3, 2, x, pb, pm))
        for b in range(n):
            sign = torch.from_numpy(_signs(spec, seeds[ids.index(tasks[b])], tasks[b], slots[b], cols)).cuda()
            xd = x[b].double()
            want = base @ xd + lam * (m[slots[b]] @ (xd * sign))
            y_abs = base.abs() @ xd.abs() + lam * (m[slots[b]].abs() @ xd.abs())
            assert ((y[b].double() - want).abs() <= np.sqrt(4.0 * cols + 2.0) * 2.0 ** -24 * y_abs).all(), (n, b)
    plan.close()


@pytest.mark.parametrize("x_dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_many_tokens_on_a_large_matrix(group, x_dtype):
    rng = np.random.default_rng(22)
    rows, cols = 8200, 4100
    p = randes.pack(on_gpu(weight(rng, rows, cols, wl.F32), wl.F32), group=group)
    w = p.unpack().double()
    for n in (33, 64):
        x = torch.randn(n, cols, device="cuda").to(TYPES[x_dtype])
        y = randes.packed_linear(x, p)
        want, y_abs = x.double() @ w.T, x.double().abs() @ w.abs().T
        assert ((y.double() - want).abs() <= np.sqrt(2.0 * cols + 2.0) * 2.0 ** -24 * y_abs).all(), n


@pytest.mark.parametrize("n,rows,cols", [(12, 200, 128), (40, 200, 320), (64, 2100, 192)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_many_tokens_with_extreme_activations(group, n, rows, cols):
    rng = np.random.default_rng(23)
    w = dyadic_weight(rng, rows, cols, group)
    w[w == 0] = np.float32(2.0 ** -7)                      # few zero codes: an infinity times zero is a NaN
    p = randes.pack(on_gpu(w, wl.F32), group=group)
    v = p.unpack().cpu().numpy().astype(np.float64)
    x = rng.standard_normal((n, cols)).astype(np.float32)
    x[:3] = 0
    x[0, 5] = 3e38
    x[1, 9] = 1e-30
    x[2, 7] = np.float32(1) + np.float32(2.0 ** -23)
    x[4] = 0
    x[4, 3] = np.inf
    x[5, 3] = np.nan
    x[n - 1] = 0
    x[n - 1, cols - 1] = -np.inf
    for dtype in (wl.F32, wl.BF16):
        xt = on_gpu(x, dtype)
        xs = xt.double().cpu().numpy()
        y = randes.packed_linear(xt, p).cpu().numpy()
        ordinary = [b for b in range(n) if np.isfinite(xs[b]).all()]
        assert set(ordinary) >= {1, 2, 3, 6}
        want, y_abs = xs[ordinary] @ v.T, np.abs(xs[ordinary]) @ np.abs(v).T
        assert (np.abs(y[ordinary] - want) <= np.sqrt(2.0 * cols + 2.0) * 2.0 ** -24 * y_abs).all()
        for b, c, sign in ((4, 3, 1), (n - 1, cols - 1, -1)):
            live = v[:, c] != 0
            assert np.array_equal(y[b][live], sign * np.sign(v[live, c]) * np.inf) and np.isnan(y[b][~live]).all()
        assert np.isnan(y[5]).all()
        # tokens do not see one another: zeros in place of the extreme ones leave the others' bits as they are
        calm = xt.clone()
        calm[[0, 4, 5, n - 1]] = 0
        rest = [b for b in range(n) if b not in (0, 4, 5, n - 1)]
        assert np.array_equal(y[rest], randes.packed_linear(calm, p).cpu().numpy()[rest])


@pytest.mark.parametrize("n", [3, 20, 64, 130])
@pytest.mark.parametrize("x_dtype", [wl.F32, wl.BF16])
def test_tasks_and_products_on_a_side_stream_and_in_a_graph(x_dtype, n):
    rows, cols, lam = 600, 512, 0.25
    plan, spec, ids, seeds = _plan(rows, cols, 5, S | F, wl.BF16, wl.BF16, ids=[3, 0, 8, 77], seeds=[42, 43, 2 ** 35 + 1, 9])
    rng = np.random.default_rng(24)
    base, m = dyadic_weight(rng, rows, cols, 64), [dyadic_weight(rng, rows, cols, 64) for _ in range(5)]
    pb, pm = randes.pack(on_gpu(base, wl.F32)), randes.pack([on_gpu(v, wl.F32) for v in m])
    tasks = [ids[int(k)] for k in rng.integers(0, 4, size=n)]
    before = randes.randes_linear_giveups()
    x = on_gpu(np.zeros((n, cols)), x_dtype)
    y, plain = torch.full((n, rows), float("nan"), device="cuda"), torch.full((n, rows), float("nan"), device="cuda")

    def both():
        plan.packed_linear(tasks, lam, 3, x, pb, pm, y=y)
        randes.packed_linear(x, pb, y=plain)

    def right(acts, what):
        want, _ = _tasks_reference(spec, ids, seeds, tasks, lam, 3, acts, base.astype(np.float64), [v.astype(np.float64) for v in m])
        same_values(y.cpu().numpy(), want, what)
        same_values(plain.cpu().numpy(), acts.astype(np.float64) @ base.astype(np.float64).T, what)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(4):                                 # the activations arrive on the stream, right before the calls
            acts = dyadic_acts(rng, n, cols)
            x.copy_(on_gpu(acts, x_dtype))
            both()
    side.synchronize()
    right(acts, "side stream")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        acts = dyadic_acts(rng, n, cols)
        x.copy_(on_gpu(acts, x_dtype))
        y.fill_(float("nan"))
        plain.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        right(acts, "graph")
    assert randes.randes_linear_giveups() == before
    plan.close()
