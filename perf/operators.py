"""Workloads of the four-bit weight operators and of token scoring.

Each case is one pass through one operator as a serving or scoring program calls it:

* ``pack``      a weight matrix (or the weight retrieved from base and superposition) goes into four bits with a scale per
                group of columns, and is read back in its own type;
* ``linear``    a few tokens through one four-bit matrix;
* ``tasks``     a few tokens, each of its own task, through a four-bit base and a four-bit superposition;
* ``score``     log probabilities of given tokens, entropy and the top alternatives out of logits;
* ``train``     the same log probabilities and entropy, then the gradient with respect to the logits.

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
        dict(name="pack_proj", op="pack", rows=768, cols=768, dtype="f32", group=64, retrieved=False),
        # a language model's head over its whole vocabulary, bf16
        dict(name="pack_head", op="pack", rows=50257, cols=768, dtype="bf16", group=64, retrieved=False),
        # one large projection of one task, from base and superposition straight into four bits
        dict(name="pack_retrieved", op="pack", rows=8192, cols=4096, dtype="bf16", group=128, retrieved=True),
        # decoding one token through a small projection: a call whose latency is all that counts
        dict(name="linear_1x768", op="linear", rows=768, cols=768, group=64, tokens=1, x="bf16", y="bf16"),
        # the head for four sequences: odd number of rows, fp32 logits
        dict(name="linear_head", op="linear", rows=50257, cols=768, group=64, tokens=4, x="bf16", y="f32"),
        # one token of one task through a wide layer kept as base and superposition
        dict(name="tasks_1", op="tasks", rows=4096, cols=1024, group=32, tokens=1, n_tasks=1, n_layers=4, x="bf16", y="bf16"),
        # eight sequences of five different tasks, whose layers lie in different slots; fp32 activations
        dict(name="tasks_8_mixed", op="tasks", rows=4096, cols=4096, group=64, tokens=8, n_tasks=5, n_layers=6, x="f32", y="f32"),
        # the largest: a batch of 64 sequences of two tasks through an 8192 x 8192 layer
        dict(name="tasks_64", op="tasks", rows=8192, cols=8192, group=128, tokens=64, n_tasks=2, n_layers=2, x="bf16", y="bf16"),
        # the answer to one prompt: one row of logits
        dict(name="score_1", op="score", rows=1, vocab=32128, dtype="f32", top=8),
        # scoring a batch of texts, vocabulary of odd size
        dict(name="score_2048", op="score", rows=2048, vocab=50257, dtype="bf16", top=20),
        # a small training batch in fp32
        dict(name="train_64", op="train", rows=64, vocab=50257, dtype="f32"),
        # a full one in bf16
        dict(name="train_4096", op="train", rows=4096, vocab=32128, dtype="bf16"),
    ]


def _between(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pack", "linear", "tasks", "score", "train"])
    if op == "pack":
        cols = _between(rng, 65, 8192)
        rows = _between(rng, 32, min(50257, (32 << 20) // cols))
        retrieved = rng.random() < 0.5
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(["f32", "bf16"]), group=rng.choice([32, 64, 128]), retrieved=retrieved)
    if op in ("linear", "tasks"):
        cols = _between(rng, 200, 8192)
        rows = _between(rng, 64, min(50257, (48 << 20) // cols))
        c = dict(op=op, rows=rows, cols=cols, group=rng.choice([32, 64, 128]), tokens=_between(rng, 1, 64),
                 x=rng.choice(["f32", "bf16"]), y=rng.choice(["f32", "bf16"]))
        if op == "tasks":
            c["n_tasks"] = rng.randint(1, min(8, c["tokens"]))
            c["n_layers"] = rng.randint(1, 4)
        return c
    vocab = _between(rng, 1000, 131072)
    rows = _between(rng, 1, max(1, (96 << 20) // vocab))
    c = dict(op=op, rows=rows, vocab=vocab, dtype=rng.choice(["f32", "bf16"]))
    if op == "score":
        c["top"] = rng.randint(1, 32)
    return c


def _type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _size(name):
    return {"f32": 4, "bf16": 2}[name]


def _code(name):
    """The library's own number of an element type."""
    return {"f32": 0, "bf16": 1}[name]


def work(case):
    op = case["op"]
    if op == "pack":
        n = case["rows"] * case["cols"]
        packed = n / 2 + 2 * case["rows"] * -(-case["cols"] // case["group"])
        # the weight (or base and superposition) read, the four-bit form written, the values written
        return {"bytes": n * _size(case["dtype"]) * (3 if case["retrieved"] else 2) + packed, "flops": n * (8 if case["retrieved"] else 6)}
    if op in ("linear", "tasks"):
        n, t = case["rows"] * case["cols"], case["tokens"]
        packed = n / 2 + 2 * case["rows"] * -(-case["cols"] // case["group"])
        mats = 1
        if op == "tasks":
            mats += len(set(_slots(case)))
        products = 2 if op == "tasks" else 1
        return {"bytes": mats * packed + t * (case["cols"] * _size(case["x"]) + case["rows"] * _size(case["y"])), "flops": 2.0 * n * t * products}
    n, s = case["rows"] * case["vocab"], _size(case["dtype"])
    if op == "score":
        return {"bytes": n * s + case["rows"] * (16 + 12 * case["top"]), "flops": 6.0 * n}
    return {"bytes": 3 * n * s + case["rows"] * 24, "flops": 16.0 * n}   # logits read by each direction, gradient written


# ---- the transform: which slot a task's layer lies in and its column signs ----------------------
# Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC'11), key = the task's seed.
_SEED0 = 42


def _philox(c0, c1, c2, c3, seed):
    c = [np.asarray(v, dtype=np.uint64) & np.uint64(0xFFFFFFFF) for v in np.broadcast_arrays(c0, c1, c2, c3)]
    k0, k1, m = seed & 0xFFFFFFFF, seed >> 32, np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & m, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, -1)


def _slot(task, n_layers, layer=0):
    """Slot of the superposition that holds this layer of the task: the inverse of its shuffle."""
    sigma = list(range(n_layers))
    words = _philox(np.arange((n_layers + 3) // 4), 0, 0x5045524D, task, _SEED0 + task).reshape(-1)
    for n, k in enumerate(range(n_layers, 1, -1)):
        j = (int(words[n]) * k) >> 32
        sigma[k - 1], sigma[j] = sigma[j], sigma[k - 1]
    return sigma.index(layer)


def _signs(task, slot, cols):
    words = _philox(np.arange(-(-cols // 128)), slot, 0x5349474E, task, _SEED0 + task).reshape(-1)
    bits = (words[:, None] >> np.arange(32, dtype=np.uint64)) & np.uint64(1)
    return torch.from_numpy(1.0 - 2.0 * bits.reshape(-1)[:cols].astype(np.float32)).cuda()


def _tasks(case):
    """The task of every token: the tasks take turns."""
    return [b % case["n_tasks"] for b in range(case["tokens"])]


def _slots(case):
    return [_slot(t, case["n_layers"]) for t in range(case["n_tasks"])]


# ---- inputs -----------------------------------------------------------------------------------
def _weights(gen, rows, cols, dtype, scale):
    return (torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(dtype)


def _quantise(w, group):
    """Codes + 8 as bytes, two to a byte (even column low), and the bf16 scales of a weight."""
    rows, cols = w.shape
    n = -(-cols // group)
    p = torch.zeros(rows, n * group, device=w.device)
    p[:, :cols] = w
    p = p.view(rows, n, group)
    s = (p.abs().amax(2) / torch.full((), 7.0, device=w.device)).bfloat16()
    d = s.float()[..., None]
    q = (torch.where(d > 0, p / d, torch.zeros_like(p)).round().clamp(-7, 7) + 8).to(torch.uint8).view(rows, n * group)
    return q[:, 0::2] | (q[:, 1::2] << 4), s


def _draws(case, seed):
    """Every input of a case that is made of random numbers, the same for all who ask."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, d = case["op"], {}
    if op == "pack":
        dt = _type(case["dtype"])
        d["w"] = _weights(gen, case["rows"], case["cols"], dt, 0.02)
        if case["retrieved"]:
            d["m"] = _weights(gen, case["rows"], case["cols"], dt, 3e-3)
    elif op == "linear":
        d["w"] = _weights(gen, case["rows"], case["cols"], torch.bfloat16, 0.02)
        d["x"] = torch.randn(case["tokens"], case["cols"], generator=gen, device="cuda").to(_type(case["x"]))
    elif op == "tasks":
        d["w"] = _weights(gen, case["rows"], case["cols"], torch.bfloat16, 0.02)
        d["m"] = {l: _weights(gen, case["rows"], case["cols"], torch.bfloat16, 3e-3) for l in sorted(set(_slots(case)))}
        d["x"] = torch.randn(case["tokens"], case["cols"], generator=gen, device="cuda").to(_type(case["x"]))
    else:
        z = torch.randn(case["rows"], case["vocab"], generator=gen, device="cuda") * 2.5
        d["target"] = torch.randint(0, case["vocab"], (case["rows"],), generator=gen, device="cuda")
        # every other row is sure of its token, as a trained model mostly is
        z[::2].scatter_add_(1, d["target"][::2, None], torch.full((-(-case["rows"] // 2), 1), 9.0, device="cuda"))
        d["z"] = z.to(_type(case["dtype"]))
        if op == "train":
            d["g_lp"] = torch.randn(case["rows"], generator=gen, device="cuda") / case["rows"]
            d["g_h"] = torch.randn(case["rows"], generator=gen, device="cuda") * 0.01 / case["rows"]
    return d


LAMBDA = 0.3
SCALE = 0.8   # one over the temperature


def _plan(case, n_tasks, n_layers, storage):
    from paper_2505_11204_b200 import randes

    return randes.Plan([case["rows"]] * n_layers, [case["cols"]] * n_layers, [0] * n_layers, [SHUFFLE | FLIP],
                       storage=storage, m_dtype=storage, task_ids=range(n_tasks), seeds=[_SEED0 + t for t in range(n_tasks)])


def prepare(case, seed):
    op, s = case["op"], {"case": case}
    d = _draws(case, seed)
    if op == "pack":
        s["w"] = d["w"]
        if case["retrieved"]:
            s["m"], s["sign"] = d["m"], _signs(0, 0, case["cols"])
            if own:
                s["plan"] = _plan(case, 1, 1, _code(case["dtype"]))
                s["M"] = s["plan"].new_superposition()
                s["plan"].slot(s["M"], 0).copy_(d["m"])
    elif op == "linear":
        s["x"] = d["x"]
        if own:
            from paper_2505_11204_b200 import randes

            s["packed"] = randes.pack(d["w"], group=case["group"])
        else:
            s["codes"], s["scales"] = _quantise(d["w"], case["group"])
    elif op == "tasks":
        s["x"], s["tasks"] = d["x"], _tasks(case)
        if own:
            from paper_2505_11204_b200 import randes

            s["plan"] = _plan(case, case["n_tasks"], case["n_layers"], 1)
            s["base"] = randes.pack(d["w"], group=case["group"])
            s["packed_m"] = [randes.pack(d["m"][l], group=case["group"]) if l in d["m"] else None for l in range(case["n_layers"])]
        else:
            s["codes"], s["scales"] = _quantise(d["w"], case["group"])
            s["m"] = {l: _quantise(w, case["group"]) for l, w in d["m"].items()}
            s["slot"] = _slots(case)
            s["sign"] = torch.stack([_signs(t, s["slot"][t], case["cols"]) for t in range(case["n_tasks"])])
            s["of"] = {l: torch.tensor([b for b, t in enumerate(s["tasks"]) if s["slot"][t] == l], device="cuda") for l in d["m"]}
            s["task"] = torch.tensor(s["tasks"], device="cuda")
    else:
        s.update(d)
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
            p = s["plan"].retrieve_packed(0, LAMBDA, [s["w"]], s["M"], group=case["group"])[0]
        else:
            p = randes.pack(s["w"], group=case["group"])
        return p.unpack(out_dtype=_code(case["dtype"]))
    if op == "linear":
        return randes.packed_linear(s["x"], s["packed"], y_dtype=_code(case["y"]))
    if op == "tasks":
        return s["plan"].packed_linear(s["tasks"], LAMBDA, 0, s["x"], s["base"], s["packed_m"], y_dtype=_code(case["y"]))
    if op == "score":
        r = randes.token_scores(s["z"], s["target"], top_k=case["top"], scale=SCALE)
        return {"logprob": r.logprob, "entropy": r.entropy, "ids": r.top_ids, "tops": r.top_logprobs}
    r = randes.token_scores(s["z"], s["target"], scale=SCALE)
    dz = randes.token_scores_backward(s["z"], s["target"], r, s["g_lp"], s["g_h"], scale=SCALE)
    return {"logprob": r.logprob, "entropy": r.entropy, "dz": dz}


def _values(codes, scales, cols, group):
    """The fp32 weight that codes and scales stand for."""
    q = torch.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1).float() - 8
    return (q.view(q.shape[0], -1, group) * scales.float()[..., None]).view(q.shape[0], -1)[:, :cols]


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "pack":
        w = s["w"].float()
        if case["retrieved"]:
            w = torch.add(w, s["m"].float() * s["sign"], alpha=LAMBDA)
        codes, scales = _quantise(w, case["group"])
        return _values(codes, scales, case["cols"], case["group"]).to(s["w"].dtype)
    if op == "linear":
        y = s["x"].float() @ _values(s["codes"], s["scales"], case["cols"], case["group"]).t()
        return y.to(_type(case["y"]))
    if op == "tasks":
        x = s["x"].float()
        y = x @ _values(s["codes"], s["scales"], case["cols"], case["group"]).t()
        xs = x * s["sign"][s["task"]]
        for l, (codes, scales) in s["m"].items():
            of = s["of"][l]
            y[of] += LAMBDA * (xs[of] @ _values(codes, scales, case["cols"], case["group"]).t())
        return y.to(_type(case["y"]))
    u = s["z"].float() * SCALE
    d = u - u.amax(1, keepdim=True)
    e = d.exp()
    total = e.sum(1, keepdim=True)
    logp = d - total.log()
    p = e / total
    target = s["target"][:, None]
    out = {"logprob": logp.gather(1, target)[:, 0], "entropy": -(p * logp).sum(1)}
    if op == "score":
        # one whole number for (logit, lower index first), so that equal logits have an order
        bits = s["z"].float().view(torch.int32)
        bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = (bits << 32) + (case["vocab"] - 1 - torch.arange(case["vocab"], device=bits.device))
        out["ids"] = case["vocab"] - 1 - (key.topk(case["top"], 1).values & 0xFFFFFFFF)
        out["tops"] = logp.gather(1, out["ids"])
        return out
    dz = -s["g_lp"][:, None] * p - s["g_h"][:, None] * p * (logp + out["entropy"][:, None])
    dz.scatter_add_(1, target, s["g_lp"][:, None])
    out["dz"] = (dz * SCALE).to(s["z"].dtype)
    return out


# ---- the definition in 64 bits ------------------------------------------------------------------
def _exact_packed(w, group):
    """What four bits keep of an fp64 weight: scale = greatest magnitude of the group / 7, in bf16; codes to the nearest."""
    rows, cols = w.shape
    pad = torch.nn.functional.pad(w, (0, -cols % group)).view(rows, -1, group)
    s = (pad.abs().max(2).values / 7).bfloat16().double()[..., None]
    q = torch.where(s > 0, torch.round(pad / s), torch.zeros_like(pad))
    return (torch.clip(q, -7, 7) * s).flatten(1)[:, :cols]


def _exact_weight(w, group):
    """The fp64 weight that the codes and scales handed to a product stand for."""
    codes, scales = _quantise(w, group)
    q = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device=codes.device)
    q[:, ::2], q[:, 1::2] = codes % 16, codes // 16
    return ((q - 8) * scales.double().repeat_interleave(group, 1))[:, :w.shape[1]]


def exact(case, seed):
    d = _draws(case, seed)
    op = case["op"]
    if op == "pack":
        w = d["w"].double()
        if case["retrieved"]:
            lam = float(np.float32(LAMBDA))
            w = (w + lam * _signs(0, 0, case["cols"]).double() * d["m"].double()).float().double()   # the retrieved weight is fp32
        return _exact_packed(w, case["group"])
    if op == "linear":
        return torch.einsum("bc,rc->br", d["x"].double(), _exact_weight(d["w"], case["group"]))
    if op == "tasks":
        x, slots = d["x"].double(), _slots(case)
        y = torch.einsum("bc,rc->br", x, _exact_weight(d["w"], case["group"]))
        m = {l: _exact_weight(w, case["group"]) for l, w in d["m"].items()}
        lam = float(np.float32(LAMBDA))
        for t in range(case["n_tasks"]):
            mine = [b for b, of in enumerate(_tasks(case)) if of == t]
            y[mine] += lam * torch.einsum("bc,rc->br", x[mine] * _signs(t, slots[t], case["cols"]).double(), m[slots[t]])
        return y
    u = d["z"].double() * float(np.float32(SCALE))
    lse = torch.logsumexp(u, 1)
    p = torch.exp(u - lse[:, None])
    h = lse - (p * u).sum(1)
    rows = torch.arange(case["rows"], device="cuda")
    out = {"logprob": u[rows, d["target"]] - lse, "entropy": h}
    if op == "score":
        order = torch.sort(d["z"].double(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
        out["ids"], out["tops"] = order, torch.gather(u, 1, order) - lse[:, None]
        return out
    one = torch.zeros_like(u)
    one[rows, d["target"]] = 1
    out["dz"] = float(np.float32(SCALE)) * (d["g_lp"].double()[:, None] * (one - p) - d["g_h"].double()[:, None] * p * (u - lse[:, None] + h[:, None]))
    return out
