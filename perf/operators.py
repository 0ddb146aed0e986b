"""The operators on either side of a hop, as measured cases.

  embed      the question's words: rows of a table, scaled, one output row a
             token or pooled per question (sum, mean), and the table's gradient
  constrain  penalties for what a column has had already, biases and masks on
             the logits [n][b] of relations, entities or words, and the gradients
  pack       entity sets kept in 8 bits: e4m3 codes, an exponent a row, and back
  hop        a differentiable hop whose backward pass reads such 8-bit sets

Where ``own`` is false a pass is computed in elementary torch operations,
otherwise through the public entry points of ``paper_2002_06115_amd``.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}


def _embed(name, tokens, vocab, dim, dtype, questions=0, pool="", backward=True):
    """questions: ragged bags that the tokens are spread over (0: none, every
    token has a row of its own, scaled by sqrt(dim))."""
    return dict(name=name, op="embed", tokens=tokens, vocab=vocab, dim=dim, dtype=dtype,
                questions=questions, pool=pool, backward=backward)


def _constrain(name, rows, batch, dtype, history, bias="row", mask="bits", backward=True):
    """history: mean length of a column's history; bias: none, row (shared by
    the columns), each; mask: none, bool_row, bool, bits_row, bits."""
    return dict(name=name, op="constrain", rows=rows, batch=batch, dtype=dtype, history=history,
                bias=bias, mask=mask, backward=backward)


def _pack(name, rows, batch, x="softmax"):
    return dict(name=name, op="pack", rows=rows, batch=batch, x=x)


def _hop(name, entities, relations, triples, batch, soft=False, residual=False):
    return dict(name=name, op="hop", entities=entities, relations=relations, triples=triples,
                batch=batch, soft=soft, residual=residual)


def listed():
    return [
        # One question of nine words answered at once: the smallest call.
        _embed("embed_question_b1", 9, 43_000, 128, "fp32", questions=1, pool="mean",
               backward=False),
        # The question encoder's part of a training step: a minibatch of 128
        # questions, 128-dimensional word vectors.
        _embed("embed_questions_b128", 1_411, 50_000, 128, "fp32", questions=128, pool="mean"),
        # The input layer of a language model's training step, rows of an odd width.
        _embed("embed_tokens_bf16", 16_389, 128_000, 1_001, "bf16"),
        # The same over long documents: many repeated words, half precision.
        _embed("embed_documents_fp16", 262_144, 100_003, 512, "fp16"),
        # The relations of a hop, 18 of them, for a minibatch: two hops behind it.
        _constrain("constrain_relations_b128", 18, 128, "fp32", 2),
        # The next word of one sequence, with all that it has said so far.
        _constrain("constrain_word_b1", 32_000, 1, "bf16", 700, bias="none", backward=False),
        # The next words of eight sequences under a grammar, biases for each.
        _constrain("constrain_words_b8", 100_003, 8, "bf16", 1_900, bias="each", backward=False),
        # The answer's logits on a KB of 43 thousand entities in training, the
        # last minibatch of an epoch: the seeds are masked out.
        _constrain("constrain_answers_b93", 43_000, 93, "fp32", 3),
        # The same on a million entities, of which a type's are allowed.
        _constrain("constrain_types_b64", 1_000_000, 64, "fp32", 5, mask="bool_row"),
        # Entity sets of a million entities put away and taken back.
        _pack("pack_sets_b32", 1_000_000, 32, x="sparse"),
        # A training hop on a KB of 43 thousand entities, minibatch 128.
        _hop("hop_small_b128", 43_000, 18, 190_000, 128),
        # A residual hop on a KB of uncertain facts.
        _hop("hop_soft_b64", 1_000_000, 200, 5_000_000, 64, soft=True, residual=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed", "embed", "constrain", "constrain", "constrain", "pack",
                     "hop"])
    if op == "embed":
        dim = _log_int(rng, 3, 2_048)
        vocab = _log_int(rng, 100, min(131_072, 128_000_000 // dim))
        tokens = _log_int(rng, 1, min(262_144, 100_000_000 // dim))
        pool = rng.choice(["", "sum", "mean"])
        c = _embed("", tokens, vocab, dim, rng.choice(list(DTYPES)),
                   _log_int(rng, 1, max(1, tokens // 4)) if pool else 0, pool,
                   rng.random() < 0.7)
    elif op == "constrain":
        batch = _log_int(rng, 1, 512)
        rows = _log_int(rng, 7, min(1_000_000, 60_000_000 // batch))
        c = _constrain("", rows, batch, rng.choice(list(DTYPES)),
                       _log_int(rng, 1, min(2_000, max(1, 400_000 // batch))),
                       rng.choice(["none", "row", "each"]),
                       rng.choice(["none", "bool_row", "bool", "bits_row", "bits"]),
                       rng.random() < 0.6)
    elif op == "pack":
        batch = _log_int(rng, 1, 512)
        c = _pack("", _log_int(rng, 100, min(1_000_000, 32_000_000 // batch)), batch,
                  rng.choice(["softmax", "sparse"]))
    else:
        entities = _log_int(rng, 1_000, 500_000)
        triples = int(entities * rng.uniform(3.0, 8.0))
        batch = _log_int(rng, 1, min(256, 200_000_000 // triples))
        c = _hop("", entities, _log_int(rng, 4, 1_200), triples, batch, rng.random() < 0.4,
                 rng.random() < 0.5)
    del c["name"]
    return c


# -- inputs ------------------------------------------------------------------

def _generator(seed, what):
    return torch.Generator(device="cuda").manual_seed(seed * 1_000_003 + what)


def _zipf(n, count, gen):
    """Ids below n whose ranks follow a power law, ranks in id order."""
    lo, hi = 0.5 ** -0.05, (n + 0.5) ** -0.05
    u = torch.rand(count, device="cuda", generator=gen, dtype=torch.float64)
    return (lo + u * (hi - lo)).pow(-20.0).add(0.5).long().sub(1).clamp(0, n - 1)


def _ragged(total, parts, gen):
    """Offsets [parts + 1] that cut `total` into parts of uneven lengths, some empty."""
    cut = torch.randint(0, total + 1, (parts - 1,), device="cuda", generator=gen).sort().values
    ends = torch.tensor([0, total], device="cuda")
    return torch.cat([ends[:1], cut, ends[1:]])


def _embed_arrays(case, seed):
    gen, dt, d = _generator(seed, 1), DTYPES[case["dtype"]], case["dim"]
    a = {"table": torch.randn((case["vocab"], d), device="cuda", generator=gen).to(dt),
         "ids": _zipf(case["vocab"], case["tokens"], gen), "offsets": None,
         "scale": 1.0 if case["pool"] else math.sqrt(d)}
    rows = case["questions"] if case["pool"] else case["tokens"]
    if case["pool"]:
        a["offsets"] = _ragged(case["tokens"], rows, gen)
    if case["backward"]:
        a["dout"] = torch.randn((rows, d), device="cuda", generator=gen).to(dt)
    return a


def _pack_bits(allowed):
    """Bit i % 32 of word i // 32, int32."""
    n = allowed.shape[0]
    words = torch.zeros((-(-n // 32) * 32, *allowed.shape[1:]), dtype=torch.int64, device="cuda")
    words[:n] = allowed
    at = torch.arange(32, device="cuda").view(1, 32, *[1] * (allowed.dim() - 1))
    words = (words.view(-1, 32, *allowed.shape[1:]) << at).sum(1)
    return (words - ((words >> 31) << 32)).to(torch.int32)


def _constrain_arrays(case, seed):
    gen, n, b = _generator(seed, 2), case["rows"], case["batch"]
    a = {"z": (3 * torch.randn((n, b), device="cuda", generator=gen)).to(DTYPES[case["dtype"]])}
    total = case["history"] * b
    a["history"], a["offsets"] = _zipf(n, total, gen), _ragged(total, b, gen)
    each = lambda lo, hi: lo + (hi - lo) * torch.rand(b, device="cuda", generator=gen)  # noqa: E731
    a["repeat"], a["presence"], a["frequency"] = each(1.0, 1.6), each(0.0, 0.8), each(0.0, 0.3)
    a["bias"] = a["allowed"] = a["bits"] = None
    if case["bias"] != "none":
        a["bias"] = torch.randn((n,) if case["bias"] == "row" else (n, b), device="cuda",
                                generator=gen)
    if case["mask"] != "none":
        allowed = torch.rand((n,) if case["mask"].endswith("_row") else (n, b), device="cuda",
                             generator=gen) < 0.7
        if allowed.dim() == 2:  # a column that nothing is left to
            allowed[:, b // 2] &= b < 3
        a["allowed"] = allowed
        if case["mask"].startswith("bits"):
            a["bits"] = _pack_bits(allowed)
    if case["backward"]:
        a["dout"] = torch.randn((n, b), device="cuda", generator=gen)
    return a


def _sets(n, b, x, gen):
    if x == "sparse":
        X = 1.0 - torch.rand((n, b), device="cuda", generator=gen)
        X *= torch.rand((n, b), device="cuda", generator=gen) < 0.05
        return X / X.sum(0, keepdim=True).clamp_(min=1e-6)
    return torch.softmax(torch.randn((n, b), device="cuda", generator=gen), 0)


def _hop_arrays(case, seed):
    gen = _generator(seed, 3)
    n, m, l, b = case["entities"], case["relations"], case["triples"], case["batch"]
    a = {"s": torch.randperm(n, device="cuda", generator=gen)[_zipf(n, l, gen)],
         "r": _zipf(m, l, gen), "o": torch.randint(0, n, (l,), device="cuda", generator=gen),
         "w": 1.0 - torch.rand(l, device="cuda", generator=gen) if case["soft"] else None}
    a["X"] = _sets(n, b, "softmax", gen)
    a["R"] = torch.softmax(torch.randn((m, b), device="cuda", generator=gen), 0)
    a["dY"] = torch.randn((n, b), device="cuda", generator=gen)
    return a


def prepare(case, seed):
    op = case["op"]
    if op == "pack":
        return {"op": op, "X": _sets(case["rows"], case["batch"], case["x"], _generator(seed, 4))}
    if op == "hop":
        state = {**_hop_arrays(case, seed), **case}
        if own:  # the handle that a program keeps
            import paper_2002_06115_amd as kbf
            s, r, o = (state[k].to(torch.int32).cpu().numpy() for k in "sro")
            state["kb"] = kbf.KB(s, r, o, case["entities"], case["relations"],
                                 weight=state["w"].cpu().numpy() if case["soft"] else None)
        state["X"].requires_grad_()
        state["R"].requires_grad_()
        return state
    if op == "embed":
        state = {**_embed_arrays(case, seed), **case}
        if case["backward"]:
            state["table"].requires_grad_()
        return state
    state = {**case, **_constrain_arrays(case, seed)}
    bits, allowed = state.pop("bits"), state.pop("allowed")
    state["allowed"] = allowed if bits is None else bits
    if case["backward"]:
        state["z"].requires_grad_()
        if state["bias"] is not None:
            state["bias"].requires_grad_()
    return state


# -- a pass --------------------------------------------------------------------

def run(state):
    if own:
        return {"embed": _own_embed, "constrain": _own_constrain, "pack": _own_pack,
                "hop": _own_hop}[state["op"]](state)
    return {"embed": _plain_embed, "constrain": _plain_constrain, "pack": _plain_pack,
            "hop": _plain_hop}[state["op"]](state)


def _own_embed(st):
    from paper_2002_06115_amd import chain
    out = chain.embed(st["table"], st["ids"], st["offsets"], scale=st["scale"],
                      pool=st["pool"] or None)
    if not st["backward"]:
        return {"out": out}
    return {"out": out, "dtable": torch.autograd.grad(out, st["table"], st["dout"])[0]}


def _own_constrain(st):
    from paper_2002_06115_amd import chain
    out = chain.constrain(st["z"], bias=st["bias"], allowed=st["allowed"], history=st["history"],
                          offsets=st["offsets"], repeat=st["repeat"], presence=st["presence"],
                          frequency=st["frequency"])
    if not st["backward"]:
        return {"out": out}
    if st["bias"] is None:
        return {"out": out, "dz": torch.autograd.grad(out, st["z"], st["dout"])[0]}
    dz, dbias = torch.autograd.grad(out, (st["z"], st["bias"]), st["dout"])
    return {"out": out, "dz": dz, "dbias": dbias}


def _own_pack(st):
    import paper_2002_06115_amd as kbf
    return {"X": kbf.pack(st["X"]).unpack()}


def _own_hop(st):
    import paper_2002_06115_amd as kbf
    X, R = st["X"], st["R"]
    Y = kbf.follow_residual(st["kb"], X, R, pack=True) if st["residual"] else \
        kbf.follow(st["kb"], X, R, pack=True)
    dX, dR = torch.autograd.grad(Y, (X, R), st["dY"])
    return {"Y": Y, "dX": dX, "dR": dR}


def _sums(row, terms, rows):
    """out[row[i]] += terms[i] in 64 bits: pieces of at most 64 terms of a row
    first, then the pieces, as a frequent row has up to a million terms."""
    order = torch.argsort(row)
    row = row[order]
    new = torch.arange(row.numel(), device="cuda") % 64 == 0
    new[1:] |= row[1:] != row[:-1]
    piece = new.cumsum(0) - 1
    part = torch.zeros((row.numel() // 64 + rows + 1, terms.shape[1]), dtype=torch.float64,
                       device="cuda").index_add_(0, piece, terms[order])
    at = (torch.arange(part.shape[0], device="cuda") % rows).index_copy_(0, piece, row)
    return torch.zeros((rows, terms.shape[1]), dtype=torch.float64, device="cuda").index_add_(
        0, at, part)


@torch.no_grad()
def _plain_embed(st):
    table, ids, scale, d = st["table"], st["ids"], st["scale"], st["dim"]
    dt, bag = table.dtype, None
    if st["pool"]:
        offsets = st["offsets"]
        lengths = offsets[1:] - offsets[:-1]
        bag = torch.repeat_interleave(torch.arange(lengths.numel(), device="cuda"), lengths,
                                      output_size=ids.numel())
        each = scale / lengths.clamp(min=1).float() if st["pool"] == "mean" else \
            torch.full(lengths.shape, scale, device="cuda")
        out = torch.zeros((lengths.numel(), d), device="cuda")
        out = out.index_add_(0, bag, table[ids].float()) * each[:, None]
    else:
        out = table[ids].float() * scale
    if not st["backward"]:
        return {"out": out.to(dt)}
    g = st["dout"].float()
    g = (g * each[:, None])[bag] if st["pool"] else g * scale
    return {"out": out.to(dt), "dtable": _sums(ids, g.double(), table.shape[0]).to(dt)}


@torch.no_grad()
def _plain_constrain(st):
    z, b = st["z"].float(), st["batch"]
    lengths = st["offsets"][1:] - st["offsets"][:-1]
    column = torch.repeat_interleave(torch.arange(b, device="cuda"), lengths,
                                     output_size=st["history"].numel())
    count = torch.bincount(st["history"] * b + column, minlength=z.numel()).view(z.shape)
    had = count > 0
    factor = torch.where(had, torch.where(z > 0, 1.0 / st["repeat"], st["repeat"]), 1.0)
    out = torch.where(had & (z > 0), z / st["repeat"], z * factor)
    out = out - had * st["presence"] - count * st["frequency"]
    bias, allowed = st["bias"], st["allowed"]
    if bias is not None:
        out = out + (bias if bias.dim() == 2 else bias[:, None])
    if allowed is not None:
        if allowed.dtype == torch.int32:
            i = torch.arange(st["rows"], device="cuda")
            allowed = (allowed[i // 32] >> (i % 32).view(-1, *[1] * (allowed.dim() - 1)) & 1) > 0
        allowed = allowed if allowed.dim() == 2 else allowed[:, None]
        out = torch.where(allowed, out, -math.inf)
    if not st["backward"]:
        return {"out": out}
    g = st["dout"] if allowed is None else torch.where(allowed, st["dout"], 0.0)
    got = {"out": out, "dz": (g * factor).to(st["z"].dtype)}
    if bias is not None:
        got["dbias"] = g if bias.dim() == 2 else g.double().sum(1).float()
    return got


def _as_kept(X):
    """X as 8 bits keep it: e4m3 codes of x / 2^e, 2^e a row's smallest power of
    two with max |x| <= 448 * 2^e, but at least 2^-127."""
    mantissa, exponent = torch.frexp(X.abs().amax(1, keepdim=True))  # m in [1/2, 1)
    e = (exponent - 9 + (mantissa > 0.875)).clamp(min=-127)
    x = torch.ldexp(X.double(), -e)
    return torch.ldexp(x.float().to(torch.float8_e4m3fn).double(), e).float()


@torch.no_grad()
def _plain_pack(st):
    return {"X": _as_kept(st["X"])}


@torch.no_grad()
def _plain_hop(st):
    s, r, o, X, R, dY = st["s"], st["r"], st["o"], st["X"], st["R"], st["dY"]
    w = 1.0 if st["w"] is None else st["w"][:, None].double()
    Rl, dYl = R.double()[r] * w, dY.double()[o]
    Y, dX = _sums(o, X.double()[s] * Rl, X.shape[0]), _sums(s, dYl * Rl, X.shape[0])
    dR = _sums(r, dYl * _as_kept(X)[s] * w, R.shape[0])
    if st["residual"]:
        Y, dX = Y + X, dX + dY
    return {"Y": Y.float(), "dX": dX.float(), "dR": dR.float()}


# -- what a pass cannot do without -----------------------------------------------

def work(case):
    """Every input read once, every output written once."""
    if case["op"] == "embed":
        e, d, t = SIZES[case["dtype"]], case["dim"], case["tokens"]
        rows = case["questions"] or t
        # Rows that the tokens name, at most the table's.
        w = {"bytes": 8 * t + e * d * (min(t, case["vocab"]) + rows), "flops": d * t}
        if case["backward"]:
            w["bytes"] += 8 * t + e * d * (rows + case["vocab"])
            w["flops"] += 2 * d * t
        return w
    if case["op"] == "constrain":
        e, n, b = SIZES[case["dtype"]], case["rows"], case["batch"]
        bias = {"none": 0, "row": 4 * n, "each": 4 * n * b}[case["bias"]]
        mask = {"none": 0, "bool_row": n, "bool": n * b, "bits_row": n / 8,
                "bits": n * b / 8}[case["mask"]]
        ids = 8 * case["history"] * b
        w = {"bytes": (e + 4) * n * b + bias + mask + ids, "flops": 2 * n * b}
        if case["backward"]:
            w["bytes"] += (4 + e) * n * b + bias + mask + ids
            w["flops"] += 2 * n * b
        return w
    if case["op"] == "pack":
        n, b = case["rows"], case["batch"]
        return {"bytes": 8 * n * b + 2 * n * (b + 1), "flops": 4 * n * b}
    n, m, b, l = case["entities"], case["relations"], case["batch"], case["triples"]
    ent, rel, kept, kb = 4 * n * b, 4 * m * b, n * (b + 1), (16 if case["soft"] else 12) * l
    return {"bytes": (kb + 2 * ent + rel + kept) + (kb + 2 * ent + kept + 2 * rel),
            "flops": (9 if case["soft"] else 6) * l * b}


# -- the same in 64 bits -----------------------------------------------------------

def exact(case, seed):
    return {"embed": _exact_embed, "constrain": _exact_constrain, "pack": _exact_pack,
            "hop": _exact_hop}[case["op"]](case, seed)


def _pieces_sum(rows, out_rows, d, terms):
    """out[rows[i]] += terms(i) for all i in 64 bits, a sorted piece at a time."""
    out = torch.zeros((out_rows, d), dtype=torch.float64, device="cuda")
    order = torch.argsort(rows, stable=True)
    step = max(1, (1 << 27) // d)
    for i in range(0, order.numel(), step):
        at = order[i:i + step]
        out.index_add_(0, rows[at], terms(at))
    return out


def _exact_embed(case, seed):
    a, d = _embed_arrays(case, seed), case["dim"]
    ids, t = a["ids"], case["tokens"]
    place = torch.arange(t, device="cuda")
    weight = torch.full((t,), a["scale"], dtype=torch.float64, device="cuda")
    rows = t
    if case["pool"]:
        rows = case["questions"]
        place = torch.searchsorted(a["offsets"], place, right=True) - 1
        if case["pool"] == "mean":
            weight = weight / torch.bincount(place, minlength=rows)[place]
    got = {"out": _pieces_sum(place, rows, d, lambda i: weight[i, None] * a["table"][ids[i]].double())}
    if case["backward"]:
        got["dtable"] = _pieces_sum(ids, case["vocab"], d,
                                    lambda i: weight[i, None] * a["dout"][place[i]].double())
    return got


def _exact_constrain(case, seed):
    a, b = _constrain_arrays(case, seed), case["batch"]
    z = a["z"].double()
    theta, presence, frequency = (a[k].double() for k in ("repeat", "presence", "frequency"))
    spread = torch.searchsorted(a["offsets"], torch.arange(a["history"].numel(), device="cuda"),
                                right=True) - 1
    pairs, times = torch.unique(torch.stack([a["history"], spread]), dim=1, return_counts=True)
    i, c = pairs
    v, slope = z.clone(), torch.ones_like(z)
    slope[i, c] = torch.where(z[i, c] > 0, 1 / theta[c], theta[c])
    v[i, c] = z[i, c] * slope[i, c] - presence[c] - times * frequency[c]
    open_ = torch.ones((1, 1), dtype=torch.bool, device="cuda")
    if a["allowed"] is not None:
        open_ = a["allowed"].view(case["rows"], -1)
    if a["bias"] is not None:
        v += a["bias"].double().view(case["rows"], -1)
    got = {"out": v.masked_fill(~open_, -math.inf)}
    if case["backward"]:
        g = a["dout"].double().masked_fill(~open_, 0.0)
        got["dz"] = g * slope
        if a["bias"] is not None:
            got["dbias"] = g if case["bias"] == "each" else g.sum(1)
    return got


def _exact_kept(X):
    """Nearest multiple of the step that a code of each value's size has, ties
    to even: 8 steps to a power of two, 2^-9 the smallest."""
    X = X.double()
    top = X.abs().amax(1, keepdim=True)
    e = torch.ceil(torch.log2((top / 448).clamp(min=2.0 ** -127)))
    x = X / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step * torch.exp2(e)


def _exact_pack(case, seed):
    return {"X": _exact_kept(_sets(case["rows"], case["batch"], case["x"], _generator(seed, 4)))}


def _exact_hop(case, seed):
    a = _hop_arrays(case, seed)
    s, r, o, X, R, dY = (a[k] for k in ("s", "r", "o", "X", "R", "dY"))
    n, m, b = case["entities"], case["relations"], case["batch"]
    w = torch.ones_like(s, dtype=torch.float64) if a["w"] is None else a["w"].double()
    kept = _exact_kept(X)
    Y = _pieces_sum(o, n, b, lambda i: w[i, None] * X[s[i]].double() * R[r[i]].double())
    dX = _pieces_sum(s, n, b, lambda i: w[i, None] * dY[o[i]].double() * R[r[i]].double())
    dR = _pieces_sum(r, m, b, lambda i: w[i, None] * kept[s[i]] * dY[o[i]].double())
    if case["residual"]:
        Y, dX = Y + X.double(), dX + dY.double()
    return {"Y": Y, "dX": dX, "dR": dR}
