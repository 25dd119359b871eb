"""The operators at both ends of a model that is trained around signatures, as cases that can be timed: tables of vectors that
turn sequences of symbols into paths, the cross entropy of a linear read-out over many classes, and the norm and clipping of
a step's gradients.

``own`` false: their plain form in elementary torch operations.  ``own`` true: the calls of the autograd module.
"""
import math

import torch

own = False

_TYPES = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f64": 8, "f32": 4, "bf16": 2, "f16": 2}


def _embed(name, N, L, D, V, dtype, grad):
    return {"name": name, "kind": "embed", "N": N, "L": L, "D": D, "V": V, "dtype": dtype, "grad": grad}


def _entropy(name, T, D, V, dtype, grad, features=False):
    return {"name": name, "kind": "entropy", "T": T, "D": D, "V": V, "dtype": dtype, "grad": grad, "features": features}


def _clip(name, layers, width, odd, dtype, out, above):
    return {"name": name, "kind": "clip", "layers": layers, "width": width, "odd": odd, "dtype": dtype, "out": out, "above": above}


def listed():
    return [
        # One symbol each of a few sequences, as they are continued: latency.
        _embed("embed_next_symbols", 8, 1, 4096, 32768, "bf16", False),
        # Sequences of symbols as paths of five channels (configuration 2's batch), trained with the kernels behind them.
        _embed("embed_paths_training", 128, 256, 5, 1000, "f64", True),
        # A training batch of a language model: 8192 tokens, a large vocabulary.
        _embed("embed_training_large", 4, 2048, 4096, 131072, "bf16", True),
        # Many tokens of a small model, some of them very frequent, an odd vocabulary.
        _embed("embed_training_frequent", 64, 4096, 1024, 50257, "f32", True),
        # The log-probability of one continuation: bound by reading the read-out.
        _entropy("entropy_score_one", 1, 4096, 32768, "bf16", False),
        # A read-out of the signatures of the benchmark's s1 (levels 0 to 6 of 4 channels: 5461 entries), doubles throughout.
        _entropy("entropy_signatures_training", 128, 5461, 1000, "f64", True, features=True),
        # A training batch in single precision.
        _entropy("entropy_training_f32", 2048, 1024, 32768, "f32", True),
        # A training batch of a middling model, an odd vocabulary and an odd number of rows.
        _entropy("entropy_training_odd", 4095, 2048, 50257, "f16", True),
        # The largest: a training batch over a large vocabulary.
        _entropy("entropy_training_large", 8192, 4096, 131072, "bf16", True),
        # The gradients of a small model around signatures: latency.
        _clip("clip_small", 2, 64, 1, "f32", "f32", True),
        # A model's gradients in bfloat16, handed to the optimizer in single precision.
        _clip("clip_large_mixed", 24, 2048, 0, "bf16", "f32", True),
        # Gradients with odd sizes throughout that stay below the bound.
        _clip("clip_odd_below", 12, 1023, 1, "f32", "f32", False),
    ]


# What a drawn case may cost: no more than the largest listed one of its kind.
_MOST_BYTES = 3.0e9
_MOST_FLOPS = {"bf16": 2.6e13, "f16": 2.6e13, "f32": 1.5e12, "f64": 5.0e11}


def _log_int(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _size(rng, low, high):
    """Round sizes as often as any: multiples of 8 or of 64 where the range has them."""
    n, step = _log_int(rng, low, high), rng.choice([1, 8, 64])
    return max(low, n // step * step) if n >= step else n


def draw(rng):
    kind = rng.choice(["embed", "entropy", "entropy", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32", "f64"])
    grad = rng.random() < 0.7
    while True:
        if kind == "embed":
            c = _embed("", _log_int(rng, 1, 128), _log_int(rng, 1, 4096), _size(rng, 2, 8192), _size(rng, 16, 262144), dtype, grad)
        elif kind == "entropy":
            c = _entropy("", _size(rng, 1, 8192), _size(rng, 8, 8192), _size(rng, 16, 262144), dtype, grad, rng.random() < 0.2)
        else:
            c = _clip("", rng.randint(1, 32), _size(rng, 8, 2048), rng.randint(0, 1), dtype, rng.choice([dtype, dtype, "f32"]),
                      rng.random() < 0.75)
        w = work(c)
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= (_MOST_FLOPS[dtype] if kind == "entropy" else math.inf):
            del c["name"]
            return c


def _clip_shapes(case):
    """The parameters of a model of `layers` layers: four square matrices, three of four times the width, two vectors; and a
    table.  odd: one entry more in every vector and one row more in every matrix."""
    w, o = case["width"], case["odd"]
    layer = [(w + o, w)] * 4 + [(4 * w + o, w)] * 3 + [(w + o,)] * 2
    return [(8 * w + o, w)] + layer * case["layers"]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = _TYPES[case["dtype"]]
    wide = torch.float64 if case["dtype"] == "f64" else torch.float32

    def randn(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, dtype=wide, device="cuda") * scale).to(dtype)

    def rand(*shape):
        return torch.rand(shape, generator=gen, dtype=torch.float64, device="cuda")

    if case["kind"] == "embed":
        N, L, V = case["N"], case["L"], case["V"]
        # Frequencies as in text: the logarithm of the rank is uniform.  Sequences end in padding, which is -1.
        tokens = (torch.exp(rand(N, L) * math.log(V)) - 1.0).long().clamp_(0, V - 1)
        ends = (rand(N, 1) * 0.2 * L).long()
        tokens = torch.where(torch.arange(L, device="cuda") < L - ends, tokens, -1)
        given = {"tokens": tokens, "table": randn(V, case["D"], scale=0.02), "scale": math.sqrt(case["D"])}
        if case["grad"]:
            given["upstream"] = randn(N, L, case["D"], scale=1e-3)
        return given
    if case["kind"] == "entropy":
        T, D, V = case["T"], case["D"], case["V"]
        h = randn(T, D)
        if case["features"]:   # features of signatures: the first is 1, those of higher levels are smaller
            h = (h.to(wide) * torch.exp(-6.0 * torch.linspace(0, 1, D, dtype=wide, device="cuda"))).to(dtype)
            h[:, 0] = 1.0
        weight = randn(V, D, scale=2.0 / math.sqrt(D))
        targets = (rand(T) * V).long().clamp_(0, V - 1)
        if T > 1:              # rows without a target: prompts and padding
            targets = torch.where(rand(T) < 0.05, -1, targets)
        return {"h": h, "weight": weight, "targets": targets}
    grads = [randn(*s, scale=1e-3 * (1 + i % 7)) for i, s in enumerate(_clip_shapes(case))]
    entries = sum(g.numel() for g in grads)
    bound = 1e-3 * math.sqrt(entries) * (0.5 if case["above"] else 50.0)
    return {"grads": grads, "bound": bound}


def prepare(case, seed):
    state = {"case": case, **_inputs(case, seed)}
    if case["kind"] == "clip":
        # the optimizer's gradients lie one behind the other
        sizes = [g.numel() for g in state["grads"]]
        state["flat"] = torch.empty(sum(sizes), dtype=_TYPES[case["out"]], device="cuda")
        state["out"] = [o.view_as(g) for o, g in zip(state["flat"].split(sizes), state["grads"])]
    elif case["grad"]:
        for name in ("table",) if case["kind"] == "embed" else ("h", "weight"):
            state[name].requires_grad_(True)
    return state


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    from paper_2509_10613_amd import autograd as ska

    case = state["case"]
    if case["kind"] == "embed":
        out = ska.embed(state["tokens"], state["table"], state["scale"])
        if not case["grad"]:
            return out
        return (out.detach(), *torch.autograd.grad(out, [state["table"]], state["upstream"]))
    if case["kind"] == "entropy":
        if not case["grad"]:
            return ska.linear_cross_entropy(state["h"], state["weight"], state["targets"], reduction="none")
        loss = ska.linear_cross_entropy(state["h"], state["weight"], state["targets"])
        return (loss.detach(), *torch.autograd.grad(loss, [state["h"], state["weight"]]))
    norm = ska.clip_grad_norm(state["grads"], state["bound"], out=state["out"])
    return norm, state["flat"]


@torch.no_grad()
def _run_plain(state):
    case = state["case"]
    dtype = _TYPES[case["dtype"]]
    wide = torch.float64 if case["dtype"] == "f64" else torch.float32
    if case["kind"] == "embed":
        tokens, table = state["tokens"], state["table"]
        V = table.shape[0]
        there = (tokens >= 0) & (tokens < V)
        at = torch.where(there, tokens, 0)
        out = torch.where(there.unsqueeze(-1), table[at].to(wide) * state["scale"], 0.0).to(dtype)
        if not case["grad"]:
            return out
        # a frequent symbol's gradient is a long sum: in 64 bits unless 16 are left of it
        sums = torch.float32 if dtype in (torch.bfloat16, torch.float16) else torch.float64
        rows = there.reshape(-1).nonzero().reshape(-1)
        grad = torch.zeros((V, case["D"]), dtype=sums, device="cuda")
        grad.index_add_(0, at.reshape(-1)[rows], state["upstream"].reshape(-1, case["D"])[rows].to(sums))
        return out, (grad * state["scale"]).to(dtype)
    if case["kind"] == "entropy":
        h, w, targets = state["h"].to(wide), state["weight"].to(wide), state["targets"]
        T, V = h.shape[0], w.shape[0]
        there = (targets >= 0) & (targets < V)
        at = torch.where(there, targets, 0)
        z = h @ w.T
        top = z.max(1, keepdim=True).values
        lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
        losses = torch.where(there, (lse - z.gather(1, at.unsqueeze(1))).squeeze(1), 0.0)
        if not case["grad"]:
            return losses
        count = there.sum().clamp(min=1)
        loss = losses.sum() / count
        g = torch.exp(z - lse)
        g[torch.arange(T, device="cuda"), at] -= 1.0
        g *= (there.to(wide) / count).unsqueeze(1)
        return loss, (g @ w).to(dtype), (g.T @ h).to(dtype)
    wide = torch.float32 if dtype in (torch.bfloat16, torch.float16) else torch.float64
    norm = torch.stack([g.double().square().sum() for g in state["grads"]]).sum().sqrt()
    factor = torch.where(torch.isfinite(norm), (state["bound"] / norm).clamp(max=1.0), 1.0).to(wide)
    for g, o in zip(state["grads"], state["out"]):
        o.copy_(g.to(wide) * factor)
    return norm, state["flat"]


@torch.no_grad()
def exact(case, seed):
    """From the definitions, in 64 bits: one row block of the classes' probabilities at a time."""
    given = _inputs(case, seed)
    if case["kind"] == "embed":
        D, V = case["D"], case["V"]
        flat = given["tokens"].reshape(-1)
        table = torch.cat([given["table"].double() * given["scale"], torch.zeros((1, D), dtype=torch.float64, device="cuda")])
        out = table[flat % (V + 1)].reshape(*given["tokens"].shape, D)   # (-1 is the row of zeros behind the last)
        if not case["grad"]:
            return out
        del table
        grad = torch.zeros((V + 1, D), dtype=torch.float64, device="cuda")
        grad.index_put_((flat % (V + 1),), given["upstream"].reshape(-1, D).double(), accumulate=True)
        return out, grad[:V] * given["scale"]
    if case["kind"] == "entropy":
        targets, V = given["targets"], case["V"]
        h, w = given["h"].double(), given["weight"].double()
        labelled = (targets >= 0).double()
        share = labelled / labelled.sum().clamp(min=1.0)
        losses, dh, dw = [], [], torch.zeros_like(w) if case["grad"] else None
        rows = max(1, (1 << 27) // V)
        for a in range(0, h.shape[0], rows):
            hb, yb = h[a:a + rows], targets[a:a + rows]
            logp = torch.log_softmax(hb @ w.T, dim=1)
            hot = torch.zeros_like(logp).scatter_(1, yb.clamp(min=0).unsqueeze(1), 1.0)
            losses.append(-(logp * hot).sum(1) * labelled[a:a + rows])
            if case["grad"]:
                g = (logp.exp_() - hot) * share[a:a + rows].unsqueeze(1)
                dh.append(g @ w)
                dw += g.T @ hb
        losses = torch.cat(losses)
        return (torch.dot(losses, share), torch.cat(dh), dw) if case["grad"] else losses
    total = 0.0
    for g in given["grads"]:
        total = total + torch.linalg.vector_norm(g, dtype=torch.float64) ** 2
    norm = total ** 0.5
    return norm, torch.cat([g.double().reshape(-1) for g in given["grads"]]) * min(1.0, given["bound"] / float(norm))


def work(case):
    """Each input read once and each output written once (of a table that is looked up, the rows); the products of the logits and of both gradients."""
    b = _BYTES[case["dtype"]]
    if case["kind"] == "embed":
        n, D, V = case["N"] * case["L"], case["D"], case["V"]
        moved = 8 * n + b * D * (min(n, V) + n)
        flops = n * D
        if case["grad"]:
            moved, flops = moved + b * D * (n + V), 2 * flops
        return {"bytes": float(moved), "flops": float(flops)}
    if case["kind"] == "entropy":
        T, D, V = case["T"], case["D"], case["V"]
        moved = b * (T * D + V * D) * (2 if case["grad"] else 1) + 8 * T
        return {"bytes": float(moved), "flops": 2.0 * T * D * V * (3 if case["grad"] else 1)}
    entries = sum(math.prod(s) for s in _clip_shapes(case))
    return {"bytes": float(entries * (b + _BYTES[case["out"]])), "flops": 3.0 * entries}
