"""Workloads of weights and activations in eight bits, products of them, and the root-mean-square norm that feeds them.

Each case is one pass through one operator as a serving or a training program calls it:

* ``pack``      a weight matrix (or the weight retrieved from base and superposition) goes into eight bits with a scale per
                128 columns, and is read back in bf16;
* ``norm``      the residual's addition and the norm of every row, its output in the activations' type or in eight bits;
* ``linear``    activations through a weight kept in eight bits, from one token to thousands;
* ``prompt``    the norm with its output in eight bits, and the product with a layer's weight right behind it;
* ``back``      backward through the norm, from the checkpoint of its input in eight bits;
* ``train``     backward through a linear layer, from the checkpoint of its input in eight bits.

With ``own`` false ``run`` computes the definition with elementary torch operations in fp32; with ``own`` true it calls the
library.  ``exact`` gives the same results in fp64.
"""
import math

import numpy as np
import torch

own = False

SHUFFLE, FLIP = 1, 2


# ---- cases ------------------------------------------------------------------------------------
def listed():
    return [
        # one attention projection of a 768-wide model, fp32 weights: the smallest matrix anyone packs
        dict(name="pack_proj", op="pack", rows=768, cols=768, dtype="f32", retrieved=False),
        # one large projection of one task, from base and superposition straight into eight bits, before a prompt is read
        dict(name="pack_retrieved", op="pack", rows=8192, cols=4096, dtype="bf16", retrieved=True),
        # decoding one token: the norm before a layer, where latency is all that counts
        dict(name="norm_1", op="norm", rows=1, cols=1024, dtype="bf16", residual=True, packed=False),
        # a ragged batch in fp32, rows of odd length, output in eight bits
        dict(name="norm_odd", op="norm", rows=777, cols=4001, dtype="f32", residual=True, packed=True),
        # a full batch of prompts
        dict(name="norm_8192", op="norm", rows=8192, cols=4096, dtype="bf16", residual=True, packed=True),
        # decoding one token through a projection
        dict(name="linear_1", op="linear", rows=4096, cols=1024, tokens=1, x="bf16", y="bf16"),
        # the vocabulary head for a batch of sequences: odd number of rows, fp32 logits
        dict(name="linear_head", op="linear", rows=50257, cols=768, tokens=48, x="bf16", y="f32"),
        # the largest: a full batch of prompts through a wide layer
        dict(name="linear_8192", op="linear", rows=8192, cols=8192, tokens=8192, x="bf16", y="bf16"),
        # one prompt of odd length through norm and projection
        dict(name="prompt_1000", op="prompt", rows=4096, cols=4096, tokens=1000, dtype="bf16"),
        # a small training batch in fp32
        dict(name="back_small", op="back", rows=200, cols=768, dtype="f32"),
        # a full one in bf16
        dict(name="back_8192", op="back", rows=8192, cols=4096, dtype="bf16"),
        # gradients of a layer's input and weight for a training batch
        dict(name="train_4096", op="train", rows=4096, cols=1024, tokens=4096, dtype="bf16"),
    ]


def _between(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pack", "norm", "linear", "prompt", "back", "train"])
    if op == "pack":
        cols = _between(rng, 65, 8192)
        rows = _between(rng, 32, min(50257, (32 << 20) // cols))
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(["f32", "bf16"]), retrieved=rng.random() < 0.5)
    if op == "norm":
        cols = _between(rng, 100, 16384)
        return dict(op=op, rows=_between(rng, 1, max(1, (32 << 20) // cols)), cols=cols, dtype=rng.choice(["f32", "bf16"]),
                    residual=rng.random() < 0.75, packed=rng.random() < 0.5)
    if op == "back":
        cols = _between(rng, 100, 16384)
        return dict(op=op, rows=_between(rng, 16, max(16, (32 << 20) // cols)), cols=cols, dtype=rng.choice(["f32", "bf16"]))
    cols = _between(rng, 200, 8192)
    rows = _between(rng, 64, min(50257, (64 << 20) // cols))
    most = min(8192, (1 << 39) // (rows * cols) // (2 if op == "train" else 1))
    if op == "linear":
        return dict(op=op, rows=rows, cols=cols, tokens=_between(rng, 1, most), x=rng.choice(["f32", "bf16"]), y=rng.choice(["f32", "bf16"]))
    return dict(op=op, rows=rows, cols=cols, tokens=_between(rng, 64, max(64, most)), dtype=rng.choice(["f32", "bf16"]))


def _type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _size(name):
    return {"f32": 4, "bf16": 2}[name]


def _code(name):
    """The library's own number of an element type."""
    return {"f32": 0, "bf16": 1}[name]


def work(case):
    op, n = case["op"], case["rows"] * case["cols"]
    eight = lambda rows, cols: rows * (cols + -(-cols // 128))      # bytes of a matrix in eight bits
    if op == "pack":
        return {"bytes": n * (_size(case["dtype"]) * (2 if case["retrieved"] else 1) + 2), "flops": n * (6 if case["retrieved"] else 4)}
    if op == "norm":
        s = _size(case["dtype"])
        return {"bytes": n * (s * (3 if case["residual"] else 1) + (2 if case["packed"] else s)) + 4 * case["cols"], "flops": 6.0 * n}
    if op == "back":
        return {"bytes": n * 3 * _size(case["dtype"]) + eight(case["rows"], case["cols"]) + 8 * case["cols"] + 4 * case["rows"], "flops": 10.0 * n}
    t = case["tokens"]
    if op == "linear":
        return {"bytes": eight(case["rows"], case["cols"]) + t * (case["cols"] * _size(case["x"]) + case["rows"] * _size(case["y"])), "flops": 2.0 * n * t}
    s = _size(case["dtype"])
    if op == "prompt":      # x and the residual read, the new residual and the product written
        return {"bytes": eight(case["rows"], case["cols"]) + t * (3 * case["cols"] * s + 2 * case["rows"]) + 4 * case["cols"], "flops": 2.0 * n * t + 6.0 * t * case["cols"]}
    # the output's gradient, checkpoint and weight read, both gradients written
    return {"bytes": t * case["rows"] * s + eight(t, case["cols"]) + eight(case["cols"], case["rows"]) + t * case["cols"] * s + 4 * n, "flops": 4.0 * n * t}


# ---- the transform: the column signs of a task (one task, one layer: the layer lies in slot 0) ----
# Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC'11), key = the task's seed.
_SEED0 = 42
LAMBDA = 0.3
EPS = 1e-6


def _signs(task, slot, cols):
    c = [np.asarray(v, dtype=np.uint64) for v in np.broadcast_arrays(np.arange(-(-cols // 128)), slot, 0x5349474E, task)]
    k0, k1, m = _SEED0 + task, 0, np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    bits = (np.stack(c, -1).reshape(-1)[:, None] >> np.arange(32, dtype=np.uint64)) & np.uint64(1)
    return torch.from_numpy(1.0 - 2.0 * bits.reshape(-1)[:cols].astype(np.float32)).cuda()


# ---- inputs -----------------------------------------------------------------------------------
def _draws(case, seed):
    """Every input of a case that is made of random numbers, the same for all who ask."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda r, c, dt, scale=1.0: (torch.randn(r, c, generator=gen, device="cuda") * scale).to(dt)
    op, rows, cols, d = case["op"], case["rows"], case["cols"], {}
    if op == "pack":
        dt = _type(case["dtype"])
        d["w"] = normal(rows, cols, dt, 0.02)
        if case["retrieved"]:
            d["m"] = normal(rows, cols, dt, 3e-3)
        return d
    if op == "linear":
        d["x"] = normal(case["tokens"], cols, _type(case["x"]))
        d["w"] = normal(rows, cols, torch.bfloat16, 0.02)
        return d
    dt = _type(case["dtype"])
    if op == "train":
        d["x"] = normal(case["tokens"], cols, dt)
        d["w"] = normal(rows, cols, torch.bfloat16, 0.02)
        d["g"] = normal(case["tokens"], rows, dt, 1e-3)
        return d
    n = rows if op in ("norm", "back") else case["tokens"]
    # a residual stream: a few of its columns are much larger than the others, as in trained models
    big = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    d["x"] = normal(n, cols, dt, 0.5)
    if case.get("residual", True):
        d["r"] = (torch.randn(n, cols, generator=gen, device="cuda") * big).to(dt)
    d["gain"] = 1 + 0.2 * torch.randn(cols, generator=gen, device="cuda")
    if op == "prompt":
        d["w"] = normal(rows, cols, torch.bfloat16, 0.02)
    if op == "back":
        d["g"], d["gh"] = normal(n, cols, dt, 1e-3), normal(n, cols, dt, 1e-3)
    return d


def prepare(case, seed):
    op, s, d = case["op"], {"case": case}, _draws(case, seed)
    if op == "pack":
        s["w"] = d["w"]
        if case["retrieved"]:
            s["m"], s["sign"] = d["m"], _signs(0, 0, case["cols"])
            if own:
                from paper_2505_11204_b200 import randes

                s["plan"] = randes.Plan([case["rows"]], [case["cols"]], [0], [SHUFFLE | FLIP], storage=_code(case["dtype"]),
                                        m_dtype=_code(case["dtype"]), task_ids=[0], seeds=[_SEED0])
                s["M"] = s["plan"].new_superposition()
                s["plan"].slot(s["M"], 0).copy_(d["m"])
        return s
    if op == "norm":
        return s | d
    if own:
        from paper_2505_11204_b200 import randes
    if op in ("linear", "prompt"):
        s |= {k: v for k, v in d.items() if k != "w"}
        s["w"] = randes.pack8(d["w"]) if own else _eight(d["w"].float())
    elif op == "train":      # the layer's weight, transposed, and the checkpoint of its input: both in eight bits
        s["g"] = d["g"]
        s["w"] = randes.pack8_transposed(d["w"]) if own else _eight(d["w"].float().t())
        s["kept"] = randes.pack8(d["x"]) if own else _eight(d["x"].float())
    else:
        s |= {k: d[k] for k in ("gain", "g", "gh")}
        if own:
            f = randes.rms_norm(d["x"], d["gain"], d["r"], eps=EPS, packed=True, checkpoint=True)
            s["kept"], s["rstd"] = f.kept, f.rstd
        else:
            h = (d["x"].float() + d["r"].float()).to(d["x"].dtype).float()
            s["kept"], s["rstd"] = _eight(h), torch.rsqrt(h.pow(2).mean(1) + EPS)
    return s


# ---- one pass ---------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2505_11204_b200 import randes

    case = s["case"]
    op = case["op"]
    if op == "pack":
        if case["retrieved"]:
            p = s["plan"].retrieve_packed8(0, LAMBDA, [s["w"]], s["M"])[0]
        else:
            p = randes.pack8(s["w"])
        return p.unpack(out_dtype=randes.BF16)
    if op == "norm":
        f = randes.rms_norm(s["x"], s["gain"], s.get("r"), eps=EPS, packed=case["packed"])
        out = {"y": f.y.unpack(out_dtype=randes.BF16) if case["packed"] else f.y, "rstd": f.rstd}
        if case["residual"]:
            out["h"] = f.h
        return out
    if op == "linear":
        return randes.packed8_linear(s["x"], s["w"], y_dtype=_code(case["y"]))
    if op == "prompt":
        f = randes.rms_norm(s["x"], s["gain"], s["r"], eps=EPS, packed=True)
        return {"h": f.h, "y": randes.packed8_linear(f.y, s["w"], y_dtype=randes.BF16)}
    if op == "back":
        dx, dgain = randes.rms_norm_backward(s["g"], s["kept"], s["rstd"], s["gain"], dh=s["gh"])
        return {"dx": dx, "dgain": dgain}
    g8, g8t = randes.pack8_both(s["g"])
    return {"dx": randes.packed8_linear(g8, s["w"], y_dtype=_code(case["dtype"])),
            "dw": randes.packed8_linear(g8t, randes.pack8_transposed(s["kept"]))}


def _eight(v):
    """Codes of an fp32 matrix (zeros up to whole blocks of 128 columns), the scale of every block, and the number of columns.
    A scale is the least power of two, 2^-100 at least, with which no element of the block is beyond 448."""
    cols = v.shape[1]
    b = torch.nn.functional.pad(v, (0, -cols % 128)).view(v.shape[0], -1, 128)
    m, e = torch.frexp(b.abs().amax(2, keepdim=True))
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-100).int()      # 448 = 0.875 * 2^9
    power = lambda k: ((k + 127) << 23).view(torch.float32)
    return (b * power(-e)).to(torch.float8_e4m3fn), power(e), cols


def _values(eight):
    """The fp32 matrix that codes and scales stand for."""
    codes, scales, cols = eight
    return (codes.float() * scales).flatten(1)[:, :cols]


def _norm(s):
    """(the new residual, one over the root mean square, the norm's output in fp32)"""
    h = s["x"].float()
    if "r" in s:
        h = (h + s["r"].float()).to(s["x"].dtype).float()      # what the program keeps is what is normed
    rstd = torch.rsqrt(h.pow(2).mean(1) + EPS)
    return h.to(s["x"].dtype), rstd, h * rstd[:, None] * s["gain"]


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "pack":
        w = s["w"].float()
        if case["retrieved"]:
            w = torch.add(w, s["m"].float() * s["sign"], alpha=LAMBDA)
        return _values(_eight(w)).bfloat16()
    if op == "norm":
        h, rstd, y = _norm(s)
        out = {"y": _values(_eight(y)).bfloat16() if case["packed"] else y.to(s["x"].dtype), "rstd": rstd}
        if case["residual"]:
            out["h"] = h
        return out
    if op == "linear":
        return (_values(_eight(s["x"].float())) @ _values(s["w"]).t()).to(_type(case["y"]))
    if op == "prompt":
        h, _, y = _norm(s)
        return {"h": h, "y": (_values(_eight(y)) @ _values(s["w"]).t()).bfloat16()}
    if op == "back":
        g, n = s["g"].float(), _values(s["kept"]) * s["rstd"][:, None]
        gg = g * s["gain"]
        dx = s["rstd"][:, None] * (gg - n * (gg * n).mean(1, keepdim=True)) + s["gh"].float()
        return {"dx": dx.to(s["g"].dtype), "dgain": (g * n).sum(0)}
    g = s["g"].float()
    dx = _values(_eight(g)) @ _values(s["w"]).t()
    dw = _values(_eight(g.t())) @ _values(_eight(_values(s["kept"]).t())).t()
    return {"dx": dx.to(s["g"].dtype), "dw": dw}


# ---- the definition in 64 bits ------------------------------------------------------------------
def _exact_eight(v):
    """What eight bits keep of an fp64 matrix: 3 bits behind the leading one, nothing below 2^-9 of the block's unit."""
    rows, cols = v.shape
    pad = torch.nn.functional.pad(v, (0, -cols % 128)).view(rows, -1, 128)
    top = pad.abs().max(2, keepdim=True).values
    unit = torch.exp2(torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -100))))
    t = pad / unit
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(t / step) * step * unit).flatten(1)[:, :cols]


def exact(case, seed):
    d, op = _draws(case, seed), case["op"]
    mul = lambda a, b: torch.einsum("nk,rk->nr", a, b)
    if op == "pack":
        w = d["w"].double()
        if case["retrieved"]:
            w = (w + float(np.float32(LAMBDA)) * _signs(0, 0, case["cols"]).double() * d["m"].double()).float().double()   # the retrieved weight is fp32
        return _exact_eight(w)
    if op == "linear":
        return mul(_exact_eight(d["x"].double()), _exact_eight(d["w"].double()))
    if op == "train":
        g, x = d["g"].double(), _exact_eight(d["x"].double())
        return {"dx": mul(_exact_eight(g), _exact_eight(d["w"].double().t())), "dw": mul(_exact_eight(g.t()), _exact_eight(x.t()))}
    h = d["x"].double()
    if "r" in d:
        h = (h + d["r"].double()).to(d["x"].dtype).double()      # the residual is kept in the activations' type
    rstd = 1 / torch.sqrt((h * h).mean(1) + EPS)
    gain = d["gain"].double()
    if op == "back":
        n, g = _exact_eight(h) * rstd[:, None], d["g"].double()
        inner = torch.einsum("nk,nk->n", g * gain, n) / case["cols"]
        return {"dx": rstd[:, None] * (g * gain - n * inner[:, None]) + d["gh"].double(), "dgain": torch.einsum("nk,nk->k", g, n)}
    y = h * rstd[:, None] * gain
    if op == "prompt":
        return {"h": h, "y": mul(_exact_eight(y), _exact_eight(d["w"].double()))}
    out = {"y": _exact_eight(y) if case["packed"] else y, "rstd": rstd}
    if case["residual"]:
        out["h"] = h
    return out
