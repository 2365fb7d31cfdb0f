"""The workloads on which the language-model operators are timed: embedding lookup with scaling, its gradient by
sorted tokens, the AdamW step over many tensors (moments in 32 or in 8 bits), and the AdamW step of the embedding rows
that a batch of tokens touched.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU from a seed, `run` makes one pass through the
operator (in its plain form, or with `own` by the library's kernels), `exact` gives the same outputs in 64 bits and
`work` the bytes and operations that no implementation can do without.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 256          # elements that share one scale of the 8-bit moments
TOP = 448.0          # largest value of the 8-bit format (e4m3)
TINY = 2.0 ** -110   # a block of first moments that stays below this is stored as zeros
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
FIRST_STEP = 10      # steps already made when a case begins
SEED = 7             # of the stochastic rounding
PADDING = -1         # the id that stands for "no token"


def listed():
    return [
        # serving: the row of the token that was just generated
        dict(name="lookup_one_token", op="lookup", V=100_000, d=512, n=1, table="float32", out="bfloat16", ids="int64",
             law="zipf", padding=0.0),
        # a short prompt, rows of an odd width in 16 bits (no row but the first starts on 4 bytes)
        dict(name="lookup_odd_rows", op="lookup", V=10_000, d=301, n=1021, table="float16", out="float16", ids="int32",
             law="uniform", padding=0.05),
        # a training batch on the large vocabulary
        dict(name="lookup_batch", op="lookup", V=1_000_000, d=300, n=65_536, table="float32", out="float32", ids="int32",
             law="zipf", padding=0.0),
        # the smallest batch, added to the gradient that the earlier micro-batches left
        dict(name="gradient_small_added", op="gradient", form="added", V=10_000, d=64, n=512, grad="float32",
             out="float32", ids="int32", law="zipf", padding=0.0),
        # a language model's whole gradient table in 16 bits, a padded batch
        dict(name="gradient_dense", op="gradient", form="dense", V=100_000, d=512, n=16_384, grad="bfloat16",
             out="bfloat16", ids="int64", law="zipf", padding=0.05),
        # the touched rows alone, as the message a data-parallel worker sends
        dict(name="gradient_rows", op="gradient", form="rows", V=1_000_000, d=300, n=65_536, grad="float32",
             out="float32", ids="int32", law="zipf", padding=0.0),
        # a small model: a few tensors of odd sizes that lie one behind the other without padding
        dict(name="adamw_small_packed", op="adamw", elements=200_003, tensors=13, packed=True, bits=32, param="float32",
             grad="float32", copy=False),
        # a large model: 32-bit weights with a 16-bit copy for the next forward pass, 16-bit gradients
        dict(name="adamw_large", op="adamw", elements=96_000_000, tensors=300, packed=False, bits=32, param="float32",
             grad="bfloat16", copy=True),
        # moments in 8 bits, a small model with 16-bit weights
        dict(name="adamw8_small", op="adamw", elements=1_000_003, tensors=25, packed=False, bits=8, param="bfloat16",
             grad="bfloat16", copy=False),
        # moments in 8 bits, a large model
        dict(name="adamw8_large", op="adamw", elements=128_000_000, tensors=300, packed=False, bits=8, param="float32",
             grad="bfloat16", copy=False),
        # one step of the medium vocabulary's rows
        dict(name="embedding_adamw_mid", op="embedding_adamw", V=100_000, d=128, n=4096, grad="float32", table="float32",
             ids="int32", law="zipf", padding=0.0),
        # one step of the large vocabulary's rows
        dict(name="embedding_adamw_large", op="embedding_adamw", V=1_000_000, d=300, n=65_536, grad="bfloat16",
             table="float32", ids="int32", law="zipf", padding=0.0),
    ]


def _log_uniform(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["lookup", "gradient", "adamw", "embedding_adamw"])
    types = ["float32", "bfloat16", "float16"]
    if op == "adamw":
        bits = rng.choice([32, 8])
        param = rng.choice(types[:2])
        return dict(op=op, elements=_log_uniform(rng, 20_000, 90_000_000), tensors=_log_uniform(rng, 1, 400),
                    packed=bits == 32 and rng.random() < 0.3, bits=bits, param=param, grad=rng.choice([param, "bfloat16"]),
                    copy=param == "float32" and rng.random() < 0.5)
    case = dict(op=op, V=_log_uniform(rng, 1000, 500_000), d=_log_uniform(rng, 16, 1024), n=_log_uniform(rng, 1, 65_536),
                ids=rng.choice(["int32", "int64"]), law=rng.choice(["zipf", "zipf", "uniform"]),
                padding=rng.choice([0.0, 0.05]))
    if rng.random() < 0.6:
        case["d"] = 8 * max(2, case["d"] // 8)
    while case["V"] * case["d"] > 100_000_000:
        case["V"] //= 2
    while case["n"] * case["d"] > 20_000_000:
        case["n"] //= 2
    if op == "lookup":
        case["table"] = rng.choice(types)
        case["out"] = rng.choice([case["table"], "bfloat16"])
    elif op == "gradient":
        case["grad"] = rng.choice(types)
        case["form"] = rng.choice(["dense", "added", "rows"])
        case["out"] = "float32" if case["form"] != "dense" else rng.choice(["float32", case["grad"]])
    else:
        case["grad"] = rng.choice(types)
        case["table"] = rng.choice(types[:2])
    return case


def _scale(case):
    return math.sqrt(case["d"])


def _sizes(case):
    """Sizes of the tensors of an AdamW case, spread over three decades as a model's matrices and vectors are."""
    r = random.Random(case["tensors"] * 1_000_003 + case["elements"])
    w = [10.0 ** r.uniform(0, 3) for _ in range(case["tensors"])]
    return [max(1, int(case["elements"] * x / sum(w))) for x in w]


def _ids(case, gen):
    u = torch.rand(case["n"], device="cuda", generator=gen, dtype=torch.float64)
    if case["law"] == "zipf":        # density 1 / rank, as the words of a text
        ids = (torch.exp(u * math.log(case["V"] + 1)) - 1).long().clamp_(0, case["V"] - 1)
    else:
        ids = (u * case["V"]).long().clamp_(0, case["V"] - 1)
    if case["padding"]:
        hole = torch.rand(case["n"], device="cuda", generator=gen) < case["padding"]
        ids = torch.where(hole, PADDING, ids)
    return ids.to(getattr(torch, case["ids"]))


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype="float32"):
        return torch.randn(*shape, device="cuda", generator=gen).mul_(std).to(getattr(torch, dtype))

    s = dict(case=case)
    if case["op"] == "adamw":
        _prepare_adamw(s, case, gen, normal)
        return s
    V, d, n = case["V"], case["d"], case["n"]
    s["ids"] = _ids(case, gen)
    if case["op"] == "lookup":
        s["table"] = normal(V, d, std=0.02, dtype=case["table"])
    else:
        s["grad"] = normal(n, d, std=1e-3, dtype=case["grad"])
    if case["op"] == "gradient" and case["form"] == "added":
        s["sum"] = normal(V, d, std=1e-3, dtype=case["out"])
    if case["op"] == "gradient" and case["form"] == "rows":      # the slot that a message is built in, and its length
        s["slot"] = (torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, d, device="cuda"),
                     torch.zeros(1, dtype=torch.int32, device="cuda"))
    if case["op"] == "embedding_adamw":
        s["table"] = normal(V, d, std=0.02, dtype=case["table"])
        s["m"] = normal(V, d, std=1e-3)
        s["v"] = normal(V, d, std=1e-3).square_()
        s["step"] = FIRST_STEP
    if own:
        from paper_2211_10280_b200 import operators

        s["embedding"] = operators.Embedding(V, d, max_tokens=n, scale=_scale(case), padding_id=PADDING)
    return s


def _prepare_adamw(s, case, gen, normal):
    sizes, at, total = _sizes(case), [], 0
    for n in sizes:
        at.append(total)
        total += n if case["packed"] else -(-n // BLOCK) * BLOCK
    real = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, n in zip(at, sizes):
        real[a:a + n] = True
    s["p"] = normal(total, std=0.02, dtype=case["param"]) * real
    s["g"] = normal(total, std=1e-3, dtype=case["grad"]) * real
    m, v = normal(total, std=3e-4) * real, normal(total, std=1e-3).square_() * real
    if case["bits"] == 8:
        m, v = m.view(-1, BLOCK), v.sqrt_().view(-1, BLOCK)
        s["m_scale"], s["v_scale"] = m.abs().amax(1) / TOP, v.amax(1) / TOP
        s["m"] = (m / s["m_scale"][:, None].clamp(min=TINY)).to(torch.float8_e4m3fn).view(-1)
        s["v"] = (v / s["v_scale"][:, None].clamp(min=TINY)).to(torch.float8_e4m3fn).view(-1)
    else:
        s["m"], s["v"] = m, v
    s["copy"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda") if case["copy"] else None
    s["step"] = FIRST_STEP
    if own:
        from paper_2211_10280_b200 import operators

        def parts(flat, unit=1):
            return None if flat is None else [flat[a // unit:a // unit - (-n // unit)] for a, n in zip(at, sizes)]

        state = dict(m=parts(s["m"]), v=parts(s["v"]))
        if case["bits"] == 8:
            state.update(m_scale=parts(s["m_scale"], BLOCK), v_scale=parts(s["v_scale"], BLOCK))
        s["grads"] = parts(s["g"])
        s["adamw"] = operators.AdamW(parts(s["p"]), lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY,
                                     state_bits=case["bits"], copies=parts(s["copy"]), state=state, step=FIRST_STEP,
                                     seed=SEED)


def run(state):
    case = state["case"]
    return {"lookup": _lookup, "gradient": _gradient, "adamw": _adamw, "embedding_adamw": _embedding_adamw}[case["op"]](
        state, case)


# ---- embedding lookup: out[i] = scale * table[ids[i]], a zero row where there is no token
def _lookup(s, case):
    out = getattr(torch, case["out"])
    if own:
        return s["embedding"].lookup(s["table"], s["ids"], dtype=out)
    rows = s["table"][s["ids"].clamp(0, case["V"] - 1)].float() * _scale(case)
    return torch.where((s["ids"] >= 0)[:, None], rows, 0.0).to(out)


# ---- its gradient: row v is scale times the sum of grad[i] over the positions i that hold v
def _summed(s, case, index, rows):
    total = torch.zeros(rows + 1, case["d"], device="cuda")
    return total.index_add_(0, index, s["grad"].float() * _scale(case))


def _touched(s, case):
    """(ids that occur, ascending, and the sums of their gradient rows)"""
    row, index = torch.unique(torch.where(s["ids"] >= 0, s["ids"], case["V"]), return_inverse=True)
    total = _summed(s, case, index, row.shape[0])
    row = row[row < case["V"]]
    return row, total[:row.shape[0]]


def _gradient(s, case):
    form, out = case["form"], getattr(torch, case["out"])
    if form == "rows":
        if own:
            s["embedding"].gradient_rows(s["grad"], s["ids"], out=s["slot"])
        else:
            row, total = _touched(s, case)
            s["slot"][0][:row.shape[0]] = row.to(torch.int32)
            s["slot"][1][:row.shape[0]] = total
            s["slot"][2].fill_(row.shape[0])
        return dict(zip(("ids", "rows", "count"), s["slot"]))
    if own:
        return s["embedding"].gradient(s["grad"], s["ids"], out=s.get("sum"), dtype=out, accumulate=form == "added")
    total = _summed(s, case, torch.where(s["ids"] >= 0, s["ids"], case["V"]).long(), case["V"])[:case["V"]]
    if form == "dense":
        return total.to(out)
    s["sum"].copy_(s["sum"].float() + total)
    return s["sum"]


# ---- AdamW: m and v the running means of the gradient and of its square,
#      p <- p (1 - lr decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
def _stepped(p, g, m, v, step):
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    root = torch.sqrt(v)
    size = LR / (1 - BETA1 ** step)
    return p * (1 - LR * DECAY) - size * (m / (root / math.sqrt(1 - BETA2 ** step) + EPS)), m, v, root


def _dither(groups, step):
    """16 random bits for each element, eight elements to a draw of Philox4x32-10 (counter: group, step, 5 << 24)."""
    low = 0xFFFFFFFF
    at = torch.arange(groups, device="cuda")
    c = [at & low, at >> 32, torch.full_like(at, step), torch.full_like(at, 5 << 24)]
    key = [SEED & low, SEED >> 32]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & low) ^ c[1] ^ key[0], b & low, ((a >> 32) & low) ^ c[3] ^ key[1], a & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    words = torch.stack(c, 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).view(-1).to(torch.int32)


def _to_8_bits(x, bits16):
    """x >= 0, at most TOP: to a neighbouring e4m3 value, the upper one as often as x is near it; subnormals to the nearest."""
    near = ((x.view(torch.int32) + (bits16 << 4) + 8) & -0x100000).view(torch.float32)
    return torch.where(x < 2.0 ** -6, x, near).clamp(max=TOP)


def _adamw(s, case):
    if own:
        s["adamw"].step(s["grads"])
    else:
        s["step"] += 1
        m, v = s["m"].float(), s["v"].float()
        if case["bits"] == 8:
            m = (m.view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
            v = (v.view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
        p, m, v, root = _stepped(s["p"].float(), s["g"].float(), m, v, s["step"])
        s["p"].copy_(p)
        if s["copy"] is not None:
            s["copy"].copy_(p)
        if case["bits"] == 8:
            bits16 = _dither(m.numel() // 8, s["step"])
            for name, x in (("m", m), ("v", root)):
                size = x.abs().view(-1, BLOCK)
                top = size.amax(1)
                top = torch.where(top < TINY, 0.0, top)
                s[name + "_scale"].copy_(top / TOP)
                size = (size * torch.where(top > 0, TOP / top, 0.0)[:, None]).view(-1)
                if name == "v":      # a positive second moment is never stored as zero
                    size = torch.where((x > 0) & (size < 2.0 ** -9), 2.0 ** -9, size)
                s[name].copy_(torch.where(x < 0, -_to_8_bits(size, bits16), _to_8_bits(size, bits16)))
        else:
            s["m"].copy_(m)
            s["v"].copy_(v)
    return {k: s[k] for k in ("p", "copy", "m", "v", "m_scale", "v_scale") if s.get(k) is not None}


# ---- the AdamW step of the rows that the batch touched; the other rows stay as they are
def _embedding_adamw(s, case):
    s["step"] += 1
    if own:
        s["embedding"].adamw(s["grad"], s["ids"], s["table"], s["m"], s["v"], step=s["step"], lr=LR, betas=(BETA1, BETA2),
                             eps=EPS, weight_decay=DECAY)
    else:
        row, total = _touched(s, case)
        row = row.long()
        p, m, v, _ = _stepped(s["table"][row].float(), total, s["m"][row], s["v"][row], s["step"])
        s["table"][row] = p.to(s["table"].dtype)
        s["m"][row] = m
        s["v"][row] = v
    return {"table": s["table"], "m": s["m"], "v": s["v"]}


# ---- the same in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s, case)
    ids, scale = s["ids"].long(), case["d"] ** 0.5
    held = ids >= 0
    if case["op"] == "lookup":
        out = torch.zeros(case["n"], case["d"], dtype=torch.float64, device="cuda")
        out[held] = s["table"][ids[held]].double() * scale
        return out
    row, index = torch.unique(ids[held], return_inverse=True)
    total = torch.zeros(row.numel(), case["d"], dtype=torch.float64, device="cuda")
    total.index_add_(0, index, s["grad"][held].double())
    total *= scale
    if case["op"] == "embedding_adamw":
        out = {k: s[k].double() for k in ("table", "m", "v")}
        t = FIRST_STEP + 1
        m = BETA1 * out["m"][row] + (1 - BETA1) * total
        v = BETA2 * out["v"][row] + (1 - BETA2) * total ** 2
        change = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + EPS)
        out["table"][row] = out["table"][row] * (1 - LR * DECAY) - LR * change
        out["m"][row], out["v"][row] = m, v
        return out
    if case["form"] == "rows":
        rows = torch.zeros(case["n"], case["d"], dtype=torch.float64, device="cuda")
        rows[:row.numel()] = total
        return {"ids": None, "rows": rows, "count": None}
    out = s["sum"].double() if case["form"] == "added" else torch.zeros(case["V"], case["d"], dtype=torch.float64, device="cuda")
    out[row] += total
    return out


def _exact_bits(groups, step):
    c = [np.arange(groups, dtype=np.uint64), np.zeros(groups, np.uint64), np.full(groups, step, np.uint64),
         np.full(groups, 5 << 24, np.uint64)]
    k0, k1 = SEED, 0
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        x, y = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(y >> half) ^ c[1] ^ np.uint64(k0), y & low, (x >> half) ^ c[3] ^ np.uint64(k1), x & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    words = np.stack(c, 1).astype(np.uint32)
    return torch.from_numpy(np.stack([words & 0xFFFF, words >> 16], 2).reshape(-1).astype(np.int32)).cuda()


def _exact_adamw(s, case):
    t = FIRST_STEP + 1
    p, g, m, v = (s[k].double() for k in ("p", "g", "m", "v"))
    if case["bits"] == 8:
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    p = p * (1 - LR * DECAY) - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + EPS)
    del g
    out = {"p": p, "m": m, "v": v}
    if case["copy"]:
        out["copy"] = p
    if case["bits"] == 8:
        share = (_exact_bits(p.numel() // 8, t).double() + 0.5) / 65536
        for name, x in (("m", m), ("v", v ** 0.5)):
            size = x.abs().view(-1, BLOCK)
            out[name + "_scale"] = size.amax(1) / TOP
            size = (size / out[name + "_scale"][:, None].clamp(min=1e-300)).view(-1)
            if name == "v":
                size = torch.where((x > 0) & (size < 2.0 ** -9), 2.0 ** -9, size)
            gap = torch.exp2(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3)
            q = torch.where(size < 2.0 ** -6, torch.round(size * 512) / 512, torch.floor(size / gap + share) * gap)
            out[name] = q.clamp(max=TOP) * torch.sign(x)
    return out


# ---- what no implementation can do without
def _bytes(name):
    return torch.empty(0, dtype=getattr(torch, name)).element_size()


def _distinct(case):
    """How many different ids a batch holds, on average."""
    rank = np.arange(case["V"], dtype=np.float64)
    p = np.log((rank + 2) / (rank + 1)) / math.log(case["V"] + 1) if case["law"] == "zipf" else np.full(case["V"], 1 / case["V"])
    return float(np.sum(-np.expm1(case["n"] * (1 - case["padding"]) * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        moments = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        each = 2 * _bytes(case["param"]) + _bytes(case["grad"]) + moments + (2 if case["copy"] else 0)
        return {"bytes": n * each, "flops": 15 * n}
    n, d, rows = case["n"], case["d"], _distinct(case)
    if case["op"] == "lookup":
        return {"bytes": n * _bytes(case["ids"]) + rows * d * _bytes(case["table"]) + n * d * _bytes(case["out"]), "flops": n * d}
    held = n * (1 - case["padding"])
    read = n * _bytes(case["ids"]) + held * d * _bytes(case["grad"])
    if case["op"] == "embedding_adamw":
        return {"bytes": read + rows * d * (2 * _bytes(case["table"]) + 16), "flops": (held + 15 * rows) * d}
    written = {"dense": case["V"] * d * _bytes(case["out"]), "added": 2 * rows * d * _bytes(case["out"]),
               "rows": rows * (d * 4 + 4)}[case["form"]]
    return {"bytes": read + written, "flops": held * d}
