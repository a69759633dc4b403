"""The operators of token models that the framework offers over plain device arrays, as measurable cases.

Three families: the AdamW step over many tensors at once (`adamw_step`, moments in 32 or in 8 bits), the log probabilities
of given tokens with their entropy and top alternatives (`log_probs`) and their gradient (`log_probs_backward`), the lookup
of embeddings with a scale (`embed`) and its gradient by sorted tokens (`embed_backward`).

`run` makes the calls of a user's program where `own` is true, and computes the same in elementary torch operations where it
is false.  `exact` computes it in 64 bits from the definitions.
"""
import math

import torch

own = False

BLOCK = 128                       # elements that share an exponent in 8-bit moments; tensors start on such a boundary
BETA1, BETA2, EPS = 0.9, 0.999, 1e-8
STEP, SEED = 37, 11               # the update's number and the seed of the rounding to 8 bits
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}


# ------------------------------------------------------------------------------------------------------------ cases
def _adamw(name, width, layers, *, bits, g="fp32", w="fp32", predict="none", clip=False):
    return dict(name=name, kind="adamw", width=width, layers=layers, bits=bits, g=g, w=w, predict=predict, clip=clip)


def _logp(name, rows, vocab, *, dtype="bf16", top=0, masked=0.0, ids="int64", scale=1.0):
    return dict(name=name, kind="logp", rows=rows, vocab=vocab, dtype=dtype, top=top, masked=masked, ids=ids, scale=scale)


def _grad(name, rows, vocab, *, dtype="bf16", entropy=False, masked=0.0, ids="int64", scale=1.0):
    return dict(name=name, kind="logp_grad", rows=rows, vocab=vocab, dtype=dtype, entropy=entropy, masked=masked, ids=ids, scale=scale)


def _embed(name, tokens, dim, vocab, *, table="bf16", out="bf16", ids="int64"):
    return dict(name=name, kind="embed", tokens=tokens, dim=dim, vocab=vocab, table=table, out=out, ids=ids)


def _embed_grad(name, tokens, dim, vocab, *, g="bf16", out="fp32", add=True, ids="int64", skew=3.0):
    return dict(name=name, kind="embed_grad", tokens=tokens, dim=dim, vocab=vocab, g=g, out=out, add=add, ids=ids, skew=skew)


def listed():
    return [
        # a small network's hundred tensors, the largest of 1024 values: bound by the calls and launches of a step
        _adamw("adamw small tensors", 16, 20, bits=32, clip=True),
        # a large model's step: 32-bit masters and moments, gradients in bf16, a bf16 copy of the predicted weights for the next pass
        _adamw("adamw 32-bit large", 2048, 6, bits=32, g="bf16", predict="bf16", clip=True),
        # a mid-sized model of odd widths with moments in 8 bits
        _adamw("adamw 8-bit odd", 511, 7, bits=8),
        # the large model where memory is short: 8-bit moments, weights and gradients in bf16
        _adamw("adamw 8-bit large", 2048, 6, bits=8, g="bf16", w="bf16"),
        # one step of one sequence: what was the token's probability, and what would the eight best have been
        _logp("logp one row", 1, 131072, top=8),
        # a batch that is being served, half of the vocabulary ruled out by a grammar, twenty alternatives reported
        _logp("logp served batch", 64, 100003, top=20, masked=0.5, scale=1.25),
        # scoring a text: entropies and log probabilities of all its tokens from 32-bit logits
        _logp("logp scoring", 4096, 32768, dtype="fp32", ids="int32"),
        # a training step's gradient over a large vocabulary
        _grad("logp gradient large", 8192, 131072),
        # the classes of an image network, with an entropy bonus: short rows of 32-bit values
        _grad("logp gradient short rows", 257, 1000, dtype="fp32", entropy=True, ids="int32"),
        # one token of each of 64 sequences
        _embed("embed one step", 64, 4096, 65536),
        # a training batch's gradient added to what the output layer left in a table that both share
        _embed_grad("embed gradient added", 8192, 1024, 50001),
        # a long batch into a gradient of its own
        _embed_grad("embed gradient whole", 131072, 1024, 65536, add=False, ids="int32"),
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, its logarithm uniform; odd as often as even."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["adamw", "logp", "logp_grad", "embed", "embed_grad"])
    ids = rng.choice(["int32", "int64"])
    if kind == "adamw":
        width = _between(rng, 16, 2048)
        layers = _between(rng, 1, max(1, min(40, int(6 * 2048 ** 2 / width ** 2))))
        c = _adamw("", width, layers, bits=rng.choice([8, 32]), g=rng.choice(["fp32", "bf16"]), w=rng.choice(["fp32", "bf16"]),
                   predict=rng.choice(["none", "fp32", "bf16"]), clip=rng.random() < 0.5)
    elif kind == "logp":
        vocab = _between(rng, 100, 200000)
        rows = _between(rng, 1, max(1, min(8192, 4096 * 32768 // vocab)))
        top = rng.choice([0, 1, 5, 20, 64]) if rows <= 512 else 0
        c = _logp("", rows, vocab, dtype=rng.choice(["fp32", "bf16"]), top=top, masked=rng.choice([0.0, 0.0, 0.3, 0.9]), ids=ids,
                  scale=rng.choice([1.0, 0.7, 1.25]))
    elif kind == "logp_grad":
        vocab = _between(rng, 100, 200000)
        rows = _between(rng, 1, max(1, min(8192, 8192 * 65536 // vocab)))
        c = _grad("", rows, vocab, dtype=rng.choice(["fp32", "bf16"]), entropy=rng.random() < 0.5, masked=rng.choice([0.0, 0.0, 0.3, 0.9]),
                  ids=ids, scale=rng.choice([1.0, 0.7, 1.25]))
    else:
        dim = _between(rng, 16, 4096)
        vocab = _between(rng, 100, min(200000, 65536 * 1024 // dim))
        tokens = _between(rng, 1, max(1, min(131072, 131072 * 1024 // dim)))
        if kind == "embed":
            c = _embed("", tokens, dim, vocab, table=rng.choice(["fp32", "bf16"]), out=rng.choice(["fp32", "bf16"]), ids=ids)
        else:
            c = _embed_grad("", tokens, dim, vocab, g=rng.choice(["fp32", "bf16"]), out=rng.choice(["fp32", "bf16"]), add=rng.random() < 0.5,
                            ids=ids, skew=rng.choice([1.0, 3.0, 6.0]))
    del c["name"]
    return c


def _shapes(case):
    """A model's tensors: a table, then for each layer two wide products, a square one, a bias and a norm's scale."""
    d = case["width"]
    return [(4 * d, d)] + [s for _ in range(case["layers"]) for s in ((4 * d, d), (d, 4 * d), (d, d), (4 * d,), (d,))]


def work(case):
    k = case["kind"]
    if k == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        # 8-bit moments come back as the values that they stand for: 8 bytes an element more
        state = 16 if case["bits"] == 32 else 4 + 4 / BLOCK + 8
        return {"bytes": n * (2 * SIZE[case["w"]] + SIZE[case["g"]] + state + SIZE.get(case["predict"], 0)), "flops": 20 * n}
    if k == "logp":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * SIZE[case["dtype"]] + case["rows"] * (28 + 12 * case["top"]), "flops": 6 * n}
    if k == "logp_grad":
        n = case["rows"] * case["vocab"]
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 28 * case["rows"], "flops": 6 * n}
    n = case["tokens"] * case["dim"]
    if k == "embed":
        return {"bytes": n * (SIZE[case["table"]] + SIZE[case["out"]]) + 8 * case["tokens"], "flops": n}
    if case["add"]:   # each row that a token names is read and written: about so many of them differ
        rows = min(case["tokens"], case["vocab"]) ** 0.9
        return {"bytes": n * SIZE[case["g"]] + 2 * rows * case["dim"] * SIZE[case["out"]], "flops": n}
    return {"bytes": n * SIZE[case["g"]] + case["vocab"] * case["dim"] * SIZE[case["out"]], "flops": n}


# ----------------------------------------------------------------------------------------------------------- inputs
def _padded(n):
    return (n + BLOCK - 1) // BLOCK * BLOCK


def _encode(x, top):
    """Codes and block exponents of moments at rest: what earlier steps of a program left (rounded to nearest here)."""
    bits = x.abs().view(torch.int32)
    e = (bits.view(-1, BLOCK).amax(1) + (1 << 20)) >> 23
    q = (bits + (1 << 19)) >> 20
    c = q - 8 * (e.repeat_interleave(BLOCK) - top)
    if top == 15:
        c = torch.where(x == 0, 0, c.clamp(0, 127)) + 128 * (x < 0)
    else:
        c = torch.where(x == 0, 0, c.clamp(1, 255))
    return c.to(torch.uint8), e.to(torch.uint8)


def _prepare_adamw(case, gen):
    def randn(n, std):
        return torch.randn(n, device="cuda", generator=gen) * std

    shapes = _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + _padded(n))
    total = starts[-1]
    real = torch.zeros(total, device="cuda")
    for n, at in zip(sizes, starts):
        real[at:at + n] = 1
    std = torch.cat([torch.full((_padded(n),), 10.0 ** (-2 - i % 3), device="cuda") for i, n in enumerate(sizes)])
    flat = (randn(total, 0.02) * real).to(DTYPE[case["w"]])
    m = randn(total, 0.3) * std * real
    v = (randn(total, 0.5).square() + 0.02) * std.square() * real
    g = randn(total, 1.0) * std
    s = {"flat": flat, "weights": [flat[at:at + n].view(sh) for sh, n, at in zip(shapes, sizes, starts)],
         "grads": [g[at:at + n].view(sh).to(DTYPE[case["g"]], copy=True) for sh, n, at in zip(shapes, sizes, starts)],
         "decay": [0.1 if len(sh) > 1 else 0.0 for sh in shapes], "sizes": sizes,
         "clip": torch.full((1,), 0.73, device="cuda") if case["clip"] else None}
    s["decay_dev"], s["padded_dev"] = torch.tensor(s["decay"], device="cuda"), torch.tensor([_padded(n) for n in sizes], device="cuda")
    del g
    if case["bits"] == 32:
        s |= {"m": m, "v": v, "m_exp": None, "v_exp": None}
    else:
        (s["m"], s["m_exp"]), (s["v"], s["v_exp"]) = _encode(m, 15), _encode(v, 31)
    if case["predict"] != "none":
        s["hat"] = torch.zeros(total, device="cuda", dtype=DTYPE[case["predict"]])
        s["predicted"] = [s["hat"][at:at + n].view(sh) for sh, n, at in zip(shapes, sizes, starts)]
    return s


def _prepare_logits(case, gen):
    rows, vocab = case["rows"], case["vocab"]
    x = torch.empty(rows, vocab, device="cuda", dtype=DTYPE[case["dtype"]])
    for at in range(0, rows, 1024):          # (a large batch piece by piece: its 32-bit values would not fit beside three states)
        y = torch.randn(min(1024, rows - at), vocab, device="cuda", generator=gen)
        y *= torch.rand(len(y), 1, device="cuda", generator=gen) * 4 + 0.5          # rows that are sure and rows that are not
        if case["masked"]:
            y.masked_fill_(torch.rand(y.shape, device="cuda", generator=gen) < case["masked"], -math.inf)
        x[at:at + len(y)] = y.to(x.dtype)
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
    if rows > 8:
        t[3::8] = -100                       # places that carry no token
        if case["masked"]:
            x[5] = -math.inf                 # nothing is left to choose from
    return x, t.to(torch.int32 if case["ids"] == "int32" else torch.int64)


def _norms(x, scale):
    """The maximum and the logarithm of the sum of a row, and its entropy, as the forward pass leaves them."""
    m, ls, h = [], [], []
    for y in x.split(512):
        y = y.double() * scale
        top = y.amax(1, keepdim=True)
        y -= torch.where(top == -math.inf, 0.0, top)
        e = y.exp()
        s = e.sum(1)
        ls.append(torch.where(s == 0, 0.0, s.log()))
        h.append(torch.where(s == 0, 0.0, s.log() - (e * y.clamp(min=-700)).sum(1) / s))
        m.append(top[:, 0])
    return torch.stack([torch.cat(m), torch.cat(ls)], 1).float(), torch.cat(h).float()


def _ids(case, gen):
    n, vocab = case["tokens"], case["vocab"]
    u = torch.rand(n, device="cuda", generator=gen, dtype=torch.float64)
    ids = (u ** case.get("skew", 1.0) * vocab).long().clamp(max=vocab - 1)
    ids = torch.randperm(vocab, device="cuda", generator=gen)[ids]      # frequent tokens lie anywhere in the table
    if n > 8:
        ids[5::64] = -1                                                 # padding
    return ids.to(torch.int32 if case["ids"] == "int32" else torch.int64)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    k = case["kind"]
    if k == "adamw":
        return {"case": case, **_prepare_adamw(case, gen)}
    s = {"case": case}
    if k in ("logp", "logp_grad"):
        s["logits"], s["targets"] = _prepare_logits(case, gen)
        if k == "logp_grad":
            s["norm"], s["entropy"] = _norms(s["logits"], case["scale"])
            n = case["rows"]
            s["g_logp"] = -(torch.rand(n, device="cuda", generator=gen) + 0.5) / n
            s["g_entropy"] = torch.randn(n, device="cuda", generator=gen) * 0.1 / n if case["entropy"] else None
        return s
    s["ids"] = _ids(case, gen)
    n, d, vocab = case["tokens"], case["dim"], case["vocab"]
    if k == "embed":
        s["table"] = (torch.randn(vocab, d, device="cuda", generator=gen) * 0.02).to(DTYPE[case["table"]])
    else:
        s["g"] = (torch.randn(n, d, device="cuda", generator=gen) * 0.01).to(DTYPE[case["g"]])
        s["table_grad"] = (torch.randn(vocab, d, device="cuda", generator=gen) * 0.01).to(DTYPE[case["out"]])
    return s


def _scale(case):
    return math.sqrt(case["dim"])


# ------------------------------------------------------------------------------------------- the framework's kernels
def _own_adamw(s):
    from paper_2003_11666_amd import adamw_moments, adamw_step
    adamw_step(s["weights"], s["grads"], s["m"], s["v"], m_exp=s["m_exp"], v_exp=s["v_exp"], step=STEP, lr=1e-3, betas=(BETA1, BETA2),
               eps=EPS, weight_decay=s["decay"], seed=SEED, grad_scale=s["clip"], predicted=s.get("predicted"), horizon=4.0)
    m, v = (s["m"], s["v"]) if s["m_exp"] is None else adamw_moments(s["m"], s["v"], s["m_exp"], s["v_exp"])
    return [s["flat"], m, v] + ([s["hat"]] if "hat" in s else [])


def _own_logp(s):
    from paper_2003_11666_amd import log_probs
    r = log_probs(s["logits"], s["targets"], scale=s["case"]["scale"], top=s["case"]["top"])
    return [r.logp, r.entropy, r.norm] + ([r.top_logp, r.top_ids] if s["case"]["top"] else [])


def _own_logp_grad(s):
    from paper_2003_11666_amd import log_probs_backward
    return log_probs_backward(s["logits"], s["targets"], s["norm"], s["g_logp"], entropy=s["entropy"], g_entropy=s["g_entropy"],
                              scale=s["case"]["scale"])


def _own_embed(s):
    from paper_2003_11666_amd import embed
    return embed(s["table"], s["ids"], scale=_scale(s["case"]), dtype=DTYPE[s["case"]["out"]])


def _own_embed_grad(s):
    from paper_2003_11666_amd import embed_backward
    return embed_backward(s["g"], s["ids"], s["table_grad"], scale=_scale(s["case"]), add=s["case"]["add"])


# ------------------------------------------------------------------------------------------------------- plain forms
GOLDEN = 0x9E3779B97F4A7C15 - (1 << 64)
MIX1, MIX2 = 0xBF58476D1CE4E5B9 - (1 << 64), 0x94D049BB133111EB - (1 << 64)


def _mix(z):
    """splitmix64's finaliser on 64-bit tensors (products wrap; a shift right brings in zeros)."""
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * MIX1
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * MIX2
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _dither(total):
    """What is added below the last bit that is kept, for m and for v: 16 random bits of each element's own, in [0, 2^20)."""
    key = _mix(SEED ^ _mix(torch.full((), STEP, dtype=torch.int64, device="cuda")))
    z = _mix(torch.arange((total + 1) // 2, device="cuda") * GOLDEN + key)
    z = torch.stack([z & 0xFFFFFFFF, (z >> 32) & 0xFFFFFFFF], 1).view(-1)[:total]
    return ((z & 0xFFFF) << 4 | 8).to(torch.int32), ((z >> 16) << 4 | 8).to(torch.int32)


def _to_codes(x, dither, top):
    bits = x.abs().view(torch.int32)
    e = (bits.view(-1, BLOCK).amax(1) + (1 << 20)) >> 23
    q = (bits + dither) >> 20
    shift = (8 * (e - top)).repeat_interleave(BLOCK)
    if top == 15:
        c = torch.where(x == 0, 0, (q - shift).clamp(0, 127)) + 128 * (x < 0)
    else:
        c = torch.where(x == 0, 0, (q.clamp(min=1) - shift).clamp(1, 255))
    return c.to(torch.uint8), e.to(torch.uint8)


def _from_codes(c, e, top):
    c, e = c.to(torch.int32), e.to(torch.int32)
    a = c & 127 if top == 15 else c
    shift = (8 * (e - top)).repeat_interleave(BLOCK)
    x = torch.where(a == 0, 0, ((a + shift).clamp(min=0) << 20)).view(torch.float32)
    x = torch.where((e == 255).repeat_interleave(BLOCK), math.nan, x)
    return torch.where(c > 127, -x, x) if top == 15 else x


def _plain_adamw(s):
    pads = torch.zeros(BLOCK, device="cuda", dtype=s["grads"][0].dtype)
    g = torch.cat([t for x, n in zip(s["grads"], s["sizes"]) for t in (x.view(-1), pads[:_padded(n) - n])]).float()
    if s["clip"] is not None:
        g = g * s["clip"]
    decay = torch.repeat_interleave(s["decay_dev"], s["padded_dev"], output_size=g.numel())
    eight = s["m_exp"] is not None
    m = _from_codes(s["m"], s["m_exp"], 15) if eight else s["m"]
    v = _from_codes(s["v"], s["v_exp"], 31) if eight else s["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g.square() * (1 - BETA2)
    lr = 1e-3
    d = lr * ((m / (1 - BETA1 ** STEP)) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS))
    w = s["flat"].float()
    w = w - lr * decay * w - d
    s["flat"].copy_(w)
    if "hat" in s:
        s["hat"].copy_(w - 4.0 * d)
    if eight:
        dm, dv = _dither(g.numel())
        for key, x, dx, top in (("m", m, dm, 15), ("v", v, dv, 31)):
            c, e = _to_codes(x, dx, top)
            s[key].copy_(c)
            s[key + "_exp"].copy_(e)
        m, v = _from_codes(s["m"], s["m_exp"], 15), _from_codes(s["v"], s["v_exp"], 31)
    else:
        m, v = s["m"].copy_(m), s["v"].copy_(v)
    return [s["flat"], m, v] + ([s["hat"]] if "hat" in s else [])


def _plain_logp(s):
    case = s["case"]
    x = s["logits"].float() * case["scale"]
    m = x.amax(1, keepdim=True)
    empty = m == -math.inf
    y = x - torch.where(empty, 0.0, m)
    e = y.exp()
    total = e.sum(1, keepdim=True)
    ls = torch.where(empty, 0.0, total.log())
    h = torch.where(empty, 0.0, ls - (e * y.clamp(min=-150)).sum(1, keepdim=True) / total)
    t = s["targets"].long()
    there = (t >= 0) & (t < case["vocab"])
    logp = torch.where(there, (y - ls).gather(1, t.clamp(0, case["vocab"] - 1)[:, None])[:, 0], 0.0)
    out = [logp, h[:, 0], torch.cat([m, ls], 1)]
    if case["top"]:
        # the largest logits, of equal ones the first: both in one 64-bit number
        bits = (s["logits"].float() + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        ids = ((order << 32) - torch.arange(case["vocab"], device="cuda")).topk(case["top"], 1).indices
        out += [(y - ls).gather(1, ids), ids.to(s["targets"].dtype)]
    return out


def _plain_logp_grad(s):
    case = s["case"]
    x = s["logits"].float() * case["scale"]
    m, ls = s["norm"][:, :1], s["norm"][:, 1:]
    empty = m == -math.inf
    lnp = x - torch.where(empty, 0.0, m) - ls
    p = lnp.exp()
    t = s["targets"].long()
    there = (t >= 0) & (t < case["vocab"])
    gl = torch.where(there, s["g_logp"], 0.0)[:, None]
    d = -gl * p
    d.scatter_add_(1, t.clamp(0, case["vocab"] - 1)[:, None], gl)
    if s["g_entropy"] is not None:
        d = d - s["g_entropy"][:, None] * p * (lnp.clamp(min=-150) + s["entropy"][:, None])
    d = torch.where(empty, 0.0, d * case["scale"])
    return d.to(s["logits"].dtype)


def _plain_embed(s):
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < s["case"]["vocab"])
    rows = s["table"][ids.clamp(0, s["case"]["vocab"] - 1)].float() * _scale(s["case"])
    return torch.where(there[:, None], rows, 0.0).to(DTYPE[s["case"]["out"]])


def _plain_embed_grad(s):
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < s["case"]["vocab"])
    g = torch.where(there[:, None], s["g"].float(), 0.0)
    total = torch.zeros(s["table_grad"].shape, device="cuda").index_add_(0, ids.clamp(0, s["case"]["vocab"] - 1), g) * _scale(s["case"])
    if s["case"]["add"]:
        total = s["table_grad"].float() + total
    return s["table_grad"].copy_(total)


def run(state):
    k = state["case"]["kind"]
    if own:
        return (_own_adamw if k == "adamw" else _own_logp if k == "logp" else _own_logp_grad if k == "logp_grad"
                else _own_embed if k == "embed" else _own_embed_grad)(state)
    return (_plain_adamw if k == "adamw" else _plain_logp if k == "logp" else _plain_logp_grad if k == "logp_grad"
            else _plain_embed if k == "embed" else _plain_embed_grad)(state)


# ------------------------------------------------------------------------------------------------------- in 64 bits
def _place(x):
    """Where |x| lies on the scale of 32-bit floats: whole steps of 2^20 units in the last place, and what is left over."""
    mant, ex = torch.frexp(x.abs())
    low = ex < -125                                             # below the smallest normal number the scale is linear
    units = torch.where(low, x.abs() * 2.0 ** 149, (mant * 2 - 1 + ex.double() + 126) * 2.0 ** 23)
    return torch.where(x == 0, 0.0, units)


def _exact_round(x, dither, top):
    u = _place(x)
    e = torch.floor((u.view(-1, BLOCK).amax(1) + 2.0 ** 20) / 2.0 ** 23).repeat_interleave(BLOCK)
    q = torch.floor((u + dither) / 2.0 ** 20)
    low = 8 * (e - top)                                         # the place of code 0, which stands for zero
    if top == 31:
        q = torch.maximum(q.clamp(min=1), low + 1)              # the second moment of a weight that has one is never zero
    q = torch.where((q <= low) | (x == 0), 0.0, q)
    ex, frac = torch.floor(q / 8), q % 8
    value = torch.where(ex == 0, frac / 8 * 2.0 ** -126, (1 + frac / 8) * 2.0 ** (ex - 127))
    return torch.where(q == 0, 0.0, value) * torch.sign(x)


def _exact_values(c, e, top):
    c, e = c.double(), e.double().repeat_interleave(BLOCK)
    sign = torch.where(c > 127, -1.0, 1.0) if top == 15 else 1.0
    a = c % 128 if top == 15 else c
    q = a + 8 * (e - top)
    ex, frac = torch.floor(q / 8), q % 8
    value = torch.where(ex <= 0, q / 8 * 2.0 ** -126, (1 + frac / 8) * 2.0 ** (ex - 127))
    return torch.where((a == 0) | (q <= 0), 0.0, value) * sign


def _in32(x):
    """A 64-bit result rounded to 32 bits: what one 32-bit operation on 32-bit operands gives."""
    return x.float().double() if isinstance(x, torch.Tensor) else float(torch.tensor(x, dtype=torch.float32))


def _exact_adamw(s, case):
    g = torch.zeros(s["flat"].numel(), dtype=torch.float64, device="cuda")
    decay = torch.zeros_like(g)
    at = 0
    for x, n, wd in zip(s["grads"], s["sizes"], s["decay"]):
        g[at:at + n] = x.double().flatten()
        decay[at:at + n] = wd
        at += _padded(n)
    if s["clip"] is not None:
        g *= s["clip"].double()
    eight = case["bits"] == 8
    m = _exact_values(s["m"], s["m_exp"], 15) if eight else s["m"].double()
    v = _exact_values(s["v"], s["v_exp"], 31) if eight else s["v"].double()
    if eight:    # moments that go into 8 bits are 32-bit values by definition, each operation rounded to them: which code one gets depends on that
        g = _in32(g)
        m = _in32(_in32(m * _in32(BETA1)) + _in32(_in32(1 - BETA1) * g))
        v = _in32(_in32(v * _in32(BETA2)) + _in32(_in32(1 - BETA2) * _in32(g * g)))
    else:
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g ** 2
    d = 1e-3 * (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
    w = s["flat"].double() * (1 - 1e-3 * decay) - d
    if eight:
        dm, dv = _dither(g.numel())
        m, v = _exact_round(m, dm.double(), 15), _exact_round(v, dv.double(), 31)
    return [w, m, v] + ([w - 4.0 * d] if "hat" in s else [])


def _exact_logp(s, case):
    logp, h, norm, tops, ids = [], [], [], [], []
    for x, t in zip(s["logits"].split(256), s["targets"].split(256)):
        z = x.double() * case["scale"]
        m = z.max(1).values
        empty = m == -math.inf
        z = z - torch.where(empty, 0.0, m)[:, None]
        p = torch.exp(z)
        total = p.sum(1)
        p /= torch.where(empty, 1.0, total)[:, None]
        ls = torch.where(empty, 0.0, torch.log(total))
        ln = z - ls[:, None]
        h.append(-(p * torch.where(p > 0, ln, 0.0)).sum(1))
        norm.append(torch.stack([m, ls], 1))
        t = t.long()
        there = (t >= 0) & (t < case["vocab"])
        logp.append(torch.where(there, ln[torch.arange(len(t), device="cuda"), t.clamp(0, case["vocab"] - 1)], 0.0))
        if case["top"]:
            first = torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
            tops.append(ln.gather(1, first))
            ids.append(first)
    out = [torch.cat(logp), torch.cat(h), torch.cat(norm)]
    return out + [torch.cat(tops), torch.cat(ids).to(s["targets"].dtype)] if case["top"] else out


def _exact_logp_grad(s, case):
    out = torch.empty(s["logits"].shape, dtype=torch.float64, device="cuda")
    for at in range(0, case["rows"], 256):
        part = slice(at, at + 256)
        z = s["logits"][part].double() * case["scale"]
        empty = (z == -math.inf).all(1)
        p = torch.softmax(z, 1)
        t = s["targets"][part].long()
        one = torch.zeros_like(p)
        there = (t >= 0) & (t < case["vocab"])
        one[torch.arange(len(t), device="cuda")[there], t[there]] = 1
        d = (s["g_logp"][part].double() * there)[:, None] * (one - p)
        if s["g_entropy"] is not None:
            ln = torch.where(p > 0, p.log(), 0.0)
            h = -(p * ln).sum(1, keepdim=True)
            d -= s["g_entropy"][part].double()[:, None] * p * (ln + h)
        out[part] = torch.where(empty[:, None], 0.0, d * case["scale"])
    return out


def _exact_embed(s, case):
    table = torch.cat([s["table"].double(), torch.zeros(1, case["dim"], dtype=torch.float64, device="cuda")])
    ids = s["ids"].long()
    return table[torch.where((ids >= 0) & (ids < case["vocab"]), ids, case["vocab"])] * _scale(case)


def _exact_embed_grad(s, case):
    ids = s["ids"].long()
    total = torch.zeros(case["vocab"] + 1, case["dim"], dtype=torch.float64, device="cuda")
    total.index_add_(0, torch.where((ids >= 0) & (ids < case["vocab"]), ids, case["vocab"]), s["g"].double())
    total = total[:-1] * _scale(case)
    return s["table_grad"].double() + total if case["add"] else total


def exact(case, seed):
    s, k = prepare(case, seed), case["kind"]
    return (_exact_adamw if k == "adamw" else _exact_logp if k == "logp" else _exact_logp_grad if k == "logp_grad"
            else _exact_embed if k == "embed" else _exact_embed_grad)(s, case)
