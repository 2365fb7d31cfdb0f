"""The workloads on which the operators of a recurrent language model are timed: layer norm and its gradient, dropout from
a counter-based generator, a gated linear recurrence with its gradient and its form for single tokens, and the draw of
the next token.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU from a seed, `run` makes one pass through the
operator (in its plain form, or with `own` by the library's kernels), `exact` gives the same outputs in 64 bits and
`work` the bytes and operations that no implementation can do without.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5           # of the layer norm
SEED = 7             # of the dropout
LOW32 = 0xFFFFFFFF


def listed():
    return [
        # serving: the row of the token that was just generated
        dict(name="norm_one_token", op="norm", direction="forward", n=1, d=512, type="bfloat16", param="float32", bias=True),
        # a ragged batch of an odd width in 16 bits
        dict(name="norm_odd_rows", op="norm", direction="forward", n=8191, d=301, type="float16", param="float16", bias=True),
        # training, the largest batch: gradients of the input, the weight and the bias
        dict(name="norm_gradient_batch", op="norm", direction="gradient", n=65_536, d=512, type="bfloat16", param="float32",
             bias=True),
        # a small batch of odd rows
        dict(name="dropout_odd", op="dropout", n=1021, d=301, type="float32", p=0.1, residual=False),
        # training, the largest batch: the end of a block, added to what the block began with
        dict(name="dropout_residual", op="dropout", n=65_536, d=512, type="bfloat16", p=0.1, residual=True),
        # serving: the next token of 64 streams, their states updated in place
        dict(name="recurrence_step", op="recurrence", direction="step", B=64, T=1, d=512, type="bfloat16", ragged=False,
             state=True, packed=True),
        # a padded batch of sentences, fp32, an odd number of steps
        dict(name="recurrence_ragged", op="recurrence", direction="forward", B=64, T=1021, d=300, type="float32", ragged=True,
             state=False, packed=False),
        # one long stream: the work has to be split along its steps
        dict(name="recurrence_long", op="recurrence", direction="forward", B=1, T=65_536, d=512, type="bfloat16", ragged=False,
             state=True, packed=True),
        # training: gradients of gates, values and first states
        dict(name="recurrence_gradient", op="recurrence", direction="gradient", B=64, T=1024, d=512, type="bfloat16",
             ragged=False, state=True, packed=False),
        # serving one stream
        dict(name="sample_one", op="sample", n=1, V=100_000, type="float32", filters="kp"),
        # many streams over the medium vocabulary, each with settings of its own
        dict(name="sample_mixed", op="sample", n=64, V=10_000, type="float32", filters="mixed"),
        # the largest batch: the mass of every token counts
        dict(name="sample_batch", op="sample", n=256, V=100_000, type="bfloat16", filters="p"),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["norm", "dropout", "recurrence", "sample"])
    kind = rng.choice(["float32", "bfloat16", "float16"])
    if op == "sample":
        V, n = _log_uniform(rng, 50, 1_000_000), _log_uniform(rng, 1, 256)
        while n * V > 12_000_000:
            n = max(1, n // 2)
        return dict(op=op, n=n, V=V, type=kind, filters=rng.choice(["none", "k", "p", "kp", "min_p", "mixed"]))
    d = _log_uniform(rng, 16, 1024)
    if rng.random() < 0.6:
        d = 8 * max(2, d // 8)
    if op == "recurrence":
        direction = rng.choice(["step", "forward", "gradient"])
        B, T = _log_uniform(rng, 1, 256), 1 if direction == "step" else _log_uniform(rng, 1, 16_384)
        while B * T * d > 16_000_000:
            if B > 1 and rng.random() < 0.5:
                B //= 2
            else:
                T = max(1, T // 2)
        return dict(op=op, direction=direction, B=B, T=T, d=d, type=kind, ragged=direction != "step" and rng.random() < 0.5,
                    state=direction == "step" or rng.random() < 0.5, packed=rng.random() < 0.5)
    n = _log_uniform(rng, 1, 65_536)
    if op == "norm":
        d = _log_uniform(rng, 16, 8192) if rng.random() < 0.3 else d
    while n * d > 16_000_000:
        n //= 2
    if op == "dropout":
        return dict(op=op, n=n, d=d, type=kind, p=rng.uniform(0.02, 0.6), residual=rng.random() < 0.5)
    return dict(op=op, direction=rng.choice(["forward", "gradient"]), n=n, d=d, type=kind,
                param=rng.choice([kind, "float32"]), bias=rng.random() < 0.7)


def _normal(gen, *shape, std=1.0, mean=0.0, dtype="float32"):
    return torch.randn(*shape, device="cuda", generator=gen).mul_(std).add_(mean).to(getattr(torch, dtype))


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    s = dict(case=case)
    {"norm": _prepare_norm, "dropout": _prepare_dropout, "recurrence": _prepare_recurrence, "sample": _prepare_sample}[case["op"]](
        s, case, gen, seed)
    return s


def _prepare_norm(s, case, gen, seed):
    n, d, kind = case["n"], case["d"], case["type"]
    # rows of the stream of a model: each with a level and a size of its own
    level, size = torch.randn(n, 1, device="cuda", generator=gen) * 0.3, torch.rand(n, 1, device="cuda", generator=gen) + 0.5
    s["x"] = (_normal(gen, n, d) * size + level).to(getattr(torch, kind))
    s["weight"] = _normal(gen, d, std=0.1, mean=1.0, dtype=case["param"])
    s["bias"] = _normal(gen, d, std=0.1, dtype=case["param"]) if case["bias"] else None
    if case["direction"] == "gradient":
        s["grad"] = _normal(gen, n, d, std=1e-2, dtype=kind)
        if own:      # what the forward pass left
            from paper_2211_10280_b200 import layers

            _, s["mean"], s["rstd"] = layers.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, stats=True)


def _prepare_dropout(s, case, gen, seed):
    s["x"] = _normal(gen, case["n"], case["d"], dtype=case["type"])
    s["residual"] = _normal(gen, case["n"], case["d"], dtype=case["type"]) if case["residual"] else None
    s["call"] = 1000 + seed % 1000


def _prepare_recurrence(s, case, gen, seed):
    B, T, d, kind = case["B"], case["T"], case["d"], case["type"]
    if case["packed"]:      # two halves of what one projection gives
        both = torch.cat([_normal(gen, B, T, d, std=2.0, mean=2.0, dtype=kind), _normal(gen, B, T, d, dtype=kind)], 2)
        s["gate"], s["value"] = both[..., :d], both[..., d:]
    else:
        s["gate"], s["value"] = _normal(gen, B, T, d, std=2.0, mean=2.0, dtype=kind), _normal(gen, B, T, d, dtype=kind)
    s["state"] = _normal(gen, B, d) if case["state"] else None
    s["lengths"] = torch.randint(1, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32) if case["ragged"] else None
    if case["direction"] == "gradient":
        s["grad"] = _normal(gen, B, T, d, std=1e-2, dtype=kind)
        s["grad_state"] = _normal(gen, B, d, std=1e-2) if case["state"] else None
        if own:      # what the forward pass left: the state before every eighth step
            from paper_2211_10280_b200 import layers

            _, _, s["marks"] = layers.recurrence(s["gate"], s["value"], s["state"], s["lengths"], marks=True)


def _prepare_sample(s, case, gen, seed):
    n, V = case["n"], case["V"]
    x = _normal(gen, n, V, std=2.5)
    few = torch.randint(0, V, (n, 8), device="cuda", generator=gen)      # what the context asks for
    x.scatter_add_(1, few, torch.rand(n, 8, device="cuda", generator=gen) * 8)
    x.masked_fill_(torch.rand(V, device="cuda", generator=gen) < 0.02, -math.inf)       # tokens that may not be drawn
    s["logits"] = x.to(getattr(torch, case["type"]))
    s["uniform"] = torch.rand(n, device="cuda", generator=gen)
    f = case["filters"]

    def pick(values, kind):
        return torch.tensor(values, device="cuda", dtype=kind)[torch.randint(0, len(values), (n,), device="cuda", generator=gen)]

    if f == "mixed":
        s["temperature"], s["top_k"] = pick([0.0, 0.6, 0.8, 1.0, 1.3], torch.float32), pick([0, 1, 20, 50, 400], torch.int32)
        s["top_p"], s["min_p"] = pick([0.5, 0.9, 0.95, 1.0], torch.float32), pick([0.0, 0.02, 0.1], torch.float32)
    else:
        s["temperature"], s["top_k"] = 0.8, 50 if "k" in f else 0
        s["top_p"], s["min_p"] = 0.9 if f in ("p", "kp") else 1.0, 0.05 if f == "min_p" else 0.0


def run(state):
    return {"norm": _norm, "dropout": _dropout, "recurrence": _recurrence, "sample": _sample}[state["case"]["op"]](
        state, state["case"])


# ---- layer norm: y = (x - mean) / sqrt(variance + eps) * weight + bias, for each row
def _norm(s, case):
    x, weight, bias = s["x"], s["weight"], s["bias"]
    if case["direction"] == "forward":
        if own:
            from paper_2211_10280_b200 import layers

            return layers.layer_norm(x, weight, bias, eps=EPS)
        c, _ = _centred(x)
        y = c * weight.float()
        return (y if bias is None else y + bias.float()).to(x.dtype)
    if own:
        from paper_2211_10280_b200 import layers

        dx, dw, db = layers.layer_norm_gradient(s["grad"], x, weight, s["mean"], s["rstd"], bias=bias is not None)
    else:
        c, r = _centred(x)
        dy = s["grad"].float()
        g = dy * weight.float()
        dx = (r * (g - g.mean(1, keepdim=True) - c * (g * c).mean(1, keepdim=True))).to(x.dtype)
        dw = (dy * c).sum(0, dtype=torch.float64).to(weight.dtype)
        db = dy.sum(0, dtype=torch.float64).to(weight.dtype)
    return {"x": dx, "weight": dw, "bias": db} if bias is not None else {"x": dx, "weight": dw}


def _centred(x):
    x = x.float()
    x = x - x.mean(1, keepdim=True)
    r = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * r, r


# ---- dropout: element e is kept where its word of Philox4x32-10 (counter: e / 4, call, 6 << 24) reaches p 2^32
def _words(groups, call):
    at = torch.arange(groups, device="cuda")
    c = [at & LOW32, at >> 32, torch.full_like(at, call & LOW32), torch.full_like(at, 6 << 24 | call >> 32)]
    key = [SEED & LOW32, SEED >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & LOW32) ^ c[1] ^ key[0], b & LOW32, ((a >> 32) & LOW32) ^ c[3] ^ key[1], a & LOW32]
        key = [(key[0] + 0x9E3779B9) & LOW32, (key[1] + 0xBB67AE85) & LOW32]
    return torch.stack(c, 1).view(-1)


def _dropout(s, case):
    x, p = s["x"], case["p"]
    if own:
        from paper_2211_10280_b200 import layers

        return layers.dropout(x, p, seed=SEED, call=s["call"], residual=s["residual"])
    kept = (_words(-(-x.numel() // 4), s["call"])[:x.numel()] >= int(p * 2 ** 32)).view_as(x)
    y = torch.where(kept, x.float() * (1 / (1 - p)), 0.0)
    return (y if s["residual"] is None else y + s["residual"].float()).to(x.dtype)


# ---- recurrence: h_t = f_t h_{t-1} + (1 - f_t) v_t with f = sigmoid(gate); steps from a sequence's length on are padding
def _scan(f, b):
    """h_t = f_t h_{t-1} + b_t along dimension 1 by doubling; overwrites both."""
    k = 1
    while k < f.shape[1]:
        b[:, k:] = b[:, k:] + f[:, k:] * b[:, :-k]
        f[:, k:] = f[:, k:] * f[:, :-k]
        k *= 2
    return b


def _parts(s, case):
    """(f, 1 - f, v, padding) in 32 bits, padded steps with f = 1, 1 - f = 0 and v = 0."""
    gate, v = s["gate"].float(), s["value"].float()
    f, rest = 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(gate))
    if s["lengths"] is None:
        return f, rest, v, None
    pad = (torch.arange(case["T"], device="cuda") >= s["lengths"][:, None])[:, :, None]
    return torch.where(pad, 1.0, f), torch.where(pad, 0.0, rest), torch.where(pad, 0.0, v), pad


def _recurrence(s, case):
    gate, value, state, lengths = s["gate"], s["value"], s["state"], s["lengths"]
    if own:
        from paper_2211_10280_b200 import layers

        if case["direction"] == "step":
            return {"out": layers.recurrence_step(gate[:, 0], value[:, 0], state), "state": state}
        if case["direction"] == "forward":
            return dict(zip(("out", "state"), layers.recurrence(gate, value, state, lengths)))
        dgate, dvalue, dstate = layers.recurrence_gradient(s["grad"], gate, value, s["marks"], lengths, grad_state=s["grad_state"])
        return {"gate": dgate, "value": dvalue, "state": dstate}
    f, rest, v, pad = _parts(s, case)
    b = rest * v
    if state is not None:
        b[:, 0] += f[:, 0] * state
    if case["direction"] == "step":
        state.copy_(b[:, 0])
        return {"out": b[:, 0].to(value.dtype), "state": state}
    if case["direction"] == "forward":
        h = _scan(f, b)
        out = h if pad is None else torch.where(pad, 0.0, h)
        return {"out": out.to(value.dtype), "state": h[:, -1].clone()}
    first = torch.zeros(case["B"], case["d"], device="cuda") if state is None else state
    before = torch.cat([first[:, None], _scan(f.clone(), b)[:, :-1]], 1)
    back = s["grad"].float()
    if pad is not None:
        back = torch.where(pad, 0.0, back)
    # D_t = dh_t + f_{t+1} D_{t+1}, from the last step to the first
    follows = torch.cat([torch.ones_like(f[:, :1]), f.flip(1)[:, :-1]], 1)
    back = back.flip(1).contiguous()
    if s["grad_state"] is not None:
        back[:, 0] += s["grad_state"]
    back = _scan(follows, back).flip(1)
    return {"gate": (f * rest * (before - v) * back).to(gate.dtype), "value": (rest * back).to(value.dtype),
            "state": f[:, 0] * back[:, 0]}


# ---- the next token: of the tokens in order (logit descending, id ascending) the first k, of those the ones with less than
#      p of the mass before them, of those the ones with at least min_p of the largest weight; then the lowest id whose running
#      weight, ids ascending, exceeds u of the whole.  A weight is exp((logit - largest) / temperature) as a multiple of 2^-bits.
#      With the token comes the logarithm of its probability among the tokens that were kept.
def _weight_bits(V):
    return min(46, 62 - (V - 1).bit_length())


def _sample(s, case):
    if own:
        from paper_2211_10280_b200 import sampling

        token, logprob = sampling.sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"],
                                         top_p=s["top_p"], min_p=s["min_p"], logprobs=True)
        return {"token": token, "logprob": logprob}
    n, V = case["n"], case["V"]

    def column(name, kind):
        x = s[name] if torch.is_tensor(s[name]) else torch.full((n,), s[name], dtype=torch.float32, device="cuda")
        return x.to(kind)[:, None]

    T, k = column("temperature", torch.float64), column("top_k", torch.int64)
    p, min_p = column("top_p", torch.float64), column("min_p", torch.float64)
    x = s["logits"].float()
    top, greedy = x.amax(1, keepdim=True), T == 0
    first = torch.where(x == top, torch.arange(V, device="cuda"), V).amin(1, keepdim=True)
    gap = x.double() - top.double()
    weight = torch.exp(gap / torch.where(greedy, 1.0, T))
    mass = torch.round(weight * 2.0 ** _weight_bits(V)).long()
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    ranked, rank = mass.gather(1, order), torch.arange(V, device="cuda")
    ranked = torch.where((k > 0) & (rank >= k), 0, ranked)
    before = ranked.cumsum(1) - ranked
    kept = ((k <= 0) | (rank < k)) & ((p >= 1) | (rank == 0) | (before.double() < p * ranked.sum(1, keepdim=True).double()))
    kept &= gap.gather(1, order) >= T * torch.log(min_p)
    running = torch.zeros_like(mass).scatter_(1, order, torch.where(kept, ranked, 0)).cumsum(1)
    total = running[:, -1:]
    target = torch.floor(s["uniform"].double()[:, None] * total.double()).long().clamp(min=0)
    token = (running <= torch.minimum(target, total - 1)).sum(1, keepdim=True)
    token = torch.where(greedy, first, token)
    logprob = gap.gather(1, token) / torch.where(greedy, 1.0, T) - torch.log(total.double() * 2.0 ** -_weight_bits(V))
    return {"token": token[:, 0], "logprob": torch.where(greedy, 0.0, logprob)[:, 0].float()}


# ---- the same in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "dropout": _exact_dropout, "recurrence": _exact_recurrence, "sample": _exact_sample}[case["op"]](s, case)


def _exact_norm(s, case):
    x, w = s["x"].double(), s["weight"].double()
    variance, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    c = (x - mean) / (variance + EPS) ** 0.5
    if case["direction"] == "forward":
        return c * w + (0 if s["bias"] is None else s["bias"].double())
    dy = s["grad"].double()
    # the product of dy with the Jacobian of each row
    g = dy * w
    g = g - (g.sum(1, keepdim=True) + c * (g * c).sum(1, keepdim=True)) / case["d"]
    out = {"x": g / (variance + EPS) ** 0.5, "weight": (dy * c).sum(0)}
    if case["bias"]:
        out["bias"] = dy.sum(0)
    return out


def _exact_dropout(s, case):
    total, call, out = s["x"].numel(), s["call"], []
    for low in range(0, -(-total // 4), 1 << 21):
        groups = min(1 << 21, -(-total // 4) - low)
        c = [np.arange(low, low + groups, dtype=np.uint64), np.zeros(groups, np.uint64), np.full(groups, call, np.uint64),
             np.full(groups, 6 << 24, np.uint64)]
        k0, k1, half, mask = SEED, 0, np.uint64(32), np.uint64(LOW32)
        for _ in range(10):
            a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
            c = [(b >> half) ^ c[1] ^ np.uint64(k0), b & mask, (a >> half) ^ c[3] ^ np.uint64(k1), a & mask]
            k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
        out.append(np.stack(c, 1).reshape(-1) >= np.uint64(math.floor(case["p"] * 2 ** 32)))
    kept = torch.from_numpy(np.concatenate(out)[:total]).cuda().view(case["n"], case["d"])
    y = s["x"].double() * kept / (1 - case["p"])
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_recurrence(s, case):
    B, T, d = case["B"], case["T"], case["d"]
    f = torch.sigmoid(s["gate"].double())
    rest, v = torch.sigmoid(-s["gate"].double()), s["value"].double()
    live = torch.ones(B, T, 1, dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        live = (torch.arange(T, device="cuda")[None] < s["lengths"][:, None])[:, :, None]
    h = torch.zeros(B, d, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    states = torch.empty(T + 1, B, d, dtype=torch.float64, device="cuda")
    states[0] = h
    drive = rest * v
    for t in range(T):
        now = torch.addcmul(drive[:, t], f[:, t], states[t])
        states[t + 1] = now if s["lengths"] is None else torch.where(live[:, t], now, states[t])
    if case["direction"] == "step":
        return {"out": states[1], "state": states[1]}
    if case["direction"] == "forward":
        return {"out": states[1:].transpose(0, 1) * live, "state": states[T]}
    carried = torch.zeros_like(h) if s["grad_state"] is None else s["grad_state"].double()
    dh = s["grad"].double()
    D = torch.zeros(B, T, d, dtype=torch.float64, device="cuda")
    for t in range(T - 1, -1, -1):
        now = dh[:, t] + carried
        D[:, t] = now if s["lengths"] is None else now * live[:, t]
        carried = f[:, t] * now if s["lengths"] is None else torch.where(live[:, t], f[:, t] * now, carried)
    return {"gate": f * rest * (states[:-1].transpose(0, 1) - v) * D, "value": rest * D, "state": carried}


def _exact_sample(s, case):
    n, V = case["n"], case["V"]
    logits, u = s["logits"].float().cpu().numpy().astype(np.float64), s["uniform"].cpu().numpy().astype(np.float64)

    def settings(name):
        x = s[name]
        return x.cpu().numpy().astype(np.float64) if torch.is_tensor(x) else np.full(n, np.float32(x), np.float64)

    T, k, p, min_p = (settings(name) for name in ("temperature", "top_k", "top_p", "min_p"))
    out, logprob = np.empty(n, np.int64), np.zeros(n)
    for i in range(n):
        x = logits[i]
        if T[i] == 0:
            out[i] = int(np.argmax(x))
            continue
        order = np.argsort(-x, kind="stable")
        if k[i] > 0:
            order = order[:int(k[i])]
        mass = np.rint(np.exp((x[order] - x[order[0]]) / T[i]) * 2.0 ** _weight_bits(V)).astype(np.int64)
        upto = np.cumsum(mass)
        if p[i] < 1:      # tokens that begin below p of the mass
            least = max(1, int(np.searchsorted((upto - mass).astype(np.float64), p[i] * float(upto[-1]), side="left")))
        else:
            least = len(order)
        order, mass = order[:least], mass[:least]
        if min_p[i] > 0:
            held = x[order] - x[order[0]] >= T[i] * math.log(min_p[i])
            order, mass = order[held], mass[held]
        by_id = np.argsort(order)
        running = np.cumsum(mass[by_id])
        out[i] = order[by_id][np.searchsorted(running, int(u[i] * float(running[-1])), side="right")]
        size = np.exp((x[order] - x[order[0]]) / T[i])
        logprob[i] = (x[out[i]] - x[order[0]]) / T[i] - math.log(size.sum())
    return {"token": torch.from_numpy(out).cuda(), "logprob": torch.from_numpy(logprob).cuda()}


# ---- what no implementation can do without
def _bytes(name):
    return torch.empty(0, dtype=getattr(torch, name)).element_size()


def work(case):
    b = _bytes(case["type"])
    if case["op"] == "sample":
        return {"bytes": case["n"] * (case["V"] * b + 4 + 8 + 4), "flops": 2 * case["n"] * case["V"]}
    if case["op"] == "recurrence":
        steps = case["B"] * case["T"] * case["d"] * (0.5 if case["ragged"] else 1.0)      # lengths are uniform
        whole, states = case["B"] * case["T"] * case["d"], case["B"] * case["d"] * 4
        if case["direction"] == "gradient":
            return {"bytes": 3 * steps * b + 2 * whole * b + states * (3 if case["state"] else 1), "flops": 16 * steps}
        return {"bytes": 2 * steps * b + whole * b + states * (2 if case["state"] else 1), "flops": 8 * steps}
    size, d = case["n"] * case["d"], case["d"]
    if case["op"] == "dropout":
        return {"bytes": size * b * (3 if case["residual"] else 2), "flops": 2 * size}
    params = d * _bytes(case["param"]) * (2 if case["bias"] else 1)
    if case["direction"] == "forward":
        return {"bytes": 2 * size * b + params, "flops": 8 * size}
    return {"bytes": 3 * size * b + params + d * _bytes(case["param"]), "flops": 16 * size}
