"""What a network of dense layers needs at its two ends and between its passes, as cases that can be timed and compared.

  checkpoint  activations kept in 8 bits: e4m3 codes, and for every 32 columns of a row a power of two that scales them
              (e8m0); encoding them, a dense layer that keeps its pre-activations so, and its backward pass from them.
  embedding   rows of a table for given tokens, times a scale; its gradient, summed over the rows of each token, for all
              rows or for each worker (group of rows) on its own.
  logprob     log probabilities of given tokens, entropy and the most probable alternatives; the gradient of the first two.

Every case has a plain form in elementary torch operations in 32 bits and, where `own` is set, the framework's calls.
"""
import math
import random

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
INT = {32: torch.int32, 64: torch.int64}
BLOCK = 32  # columns that share a scale


def listed():
    return [
        # keeping one small minibatch's activations, sizes that fit nothing
        dict(name="encode_few_odd", op="checkpoint", way="encode", dtype="fp16", rows=37, fin=1111),
        # training: the widening layer of a block, its pre-activations kept in 8 bits
        dict(name="checkpoint_fwd", op="checkpoint", way="fwd", dtype="bf16", act="gelu", rows=8192, fin=2048, fout=8192, groups=0, matrices=0, keep_x=False, x_act="none"),
        # training: its backward pass with input and pre-activations both held in 8 bits
        dict(name="checkpoint_bwd", op="checkpoint", way="bwd", dtype="bf16", act="gelu", rows=8192, fin=2048, fout=8192, groups=0, matrices=0, keep_x=True, x_act="none"),
        # 64 workers of about 128 rows on eight resident versions; the layer's input is made again from the pre-activations of the one before
        dict(name="checkpoint_versions", op="checkpoint", way="bwd", dtype="bf16", act="relu", rows=8192, fin=1568, fout=512, groups=64, matrices=8, keep_x=True, x_act="relu"),
        # serving: the tokens of a few short requests
        dict(name="embedding_few_odd", op="embedding", way="fwd", dtype="fp16", bits=64, rows=37, vocab=50257, dim=1111, groups=0, tables=0),
        # training: a whole batch's tokens, every worker's by the version it last pulled
        dict(name="embedding_versions", op="embedding", way="fwd", dtype="bf16", bits=32, rows=16384, vocab=32768, dim=2048, groups=64, tables=8),
        # training: the gradient of a large table
        dict(name="embedding_bwd", op="embedding", way="bwd", dtype="bf16", bits=64, rows=16384, vocab=50257, dim=2048, groups=0, tables=0),
        # 64 workers' own gradients, as the server buffers them
        dict(name="embedding_workers", op="embedding", way="bwd", dtype="fp32", bits=32, rows=8192, vocab=4096, dim=192, groups=64, tables=0),
        # serving: one token, with the alternatives to it
        dict(name="logprob_token", op="logprob", way="fwd", dtype="bf16", bits=64, rows=1, vocab=131072, top=20, mask=False, scale=1.25),
        # the classes of the framework's own network, for a round of 64 workers of 128 rows
        dict(name="logprob_classes", op="logprob", way="fwd", dtype="fp32", bits=64, rows=8192, vocab=10, top=0, mask=False, scale=1.0),
        # scoring given texts, an odd vocabulary with part of it masked
        dict(name="logprob_score", op="logprob", way="fwd", dtype="bf16", bits=32, rows=4096, vocab=50257, top=5, mask=True, scale=1.0),
        # training: the loss's gradient, with a bonus for entropy
        dict(name="logprob_bwd", op="logprob", way="bwd", dtype="bf16", bits=64, rows=8192, vocab=32768, top=0, mask=False, scale=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["checkpoint", "embedding", "logprob"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "checkpoint":
        way = rng.choice(["encode", "fwd", "bwd", "bwd"])
        most = 1.3e8 if way == "encode" else 1e10 if dtype == "fp32" else 1.3e11  # values, or multiply-adds
        while True:
            rows, fin, fout = _log(rng, 1, 16384), _log(rng, 32, 8192), _log(rng, 32, 8192)
            if rng.random() < 0.7:  # most layers' sizes are even ones
                fin, fout = -(-fin // 64) * 64, -(-fout // 64) * 64
            if rows * fin * (1 if way == "encode" else fout) <= most:
                break
        if way == "encode":
            return dict(op=op, way=way, dtype=dtype, rows=rows, fin=fin)
        groups = rng.choice([0, _log(rng, 2, 64)])
        while groups * fin * fout > 2e8:
            groups //= 2
        keep_x = way == "bwd" and rng.random() < 0.7
        return dict(op=op, way=way, dtype=dtype, act=rng.choice(["relu", "gelu", "silu"]), rows=rows, fin=fin, fout=fout, groups=groups,
                    matrices=rng.randint(1, groups) if groups else 0, keep_x=keep_x, x_act=rng.choice(["none", "none", "relu", "gelu", "silu"]) if keep_x else "none")
    way, bits = rng.choice(["fwd", "bwd"]), rng.choice([32, 64])
    if op == "embedding":
        groups = rng.choice([0, _log(rng, 2, 64)])
        tables = rng.randint(1, 8) if groups and way == "fwd" else 0
        while True:
            rows, vocab, dim = _log(rng, 1, 32768), _log(rng, 100, 131072), _log(rng, 16, 8192)
            if rng.random() < 0.7:
                dim = -(-dim // 64) * 64
            if rows * dim <= 3.3e7 and vocab * dim * max(1, groups if way == "bwd" else tables) <= 1e8:
                return dict(op=op, way=way, dtype=dtype, bits=bits, rows=rows, vocab=vocab, dim=dim, groups=groups, tables=tables)
    while True:
        rows, vocab = _log(rng, 1, 8192), _log(rng, 2, 262144)
        if rows * vocab <= 1.3e8:
            break
    top = rng.choice([0, 1, rng.randint(1, 32)]) if way == "fwd" else 0
    return dict(op=op, way=way, dtype=dtype, bits=bits, rows=rows, vocab=vocab, top=top, mask=rng.random() < 0.3, scale=rng.choice([1.0, 0.5, 1.25]))


# ---- inputs -------------------------------------------------------------------------------------------------------

def _split(rows, groups, seed):
    """Ragged group sizes that add up to `rows`, every eighth group empty."""
    r = random.Random(seed)
    parts = [0.0 if groups > 1 and i % 8 == 5 else 0.4 + r.random() for i in range(groups)]
    edges, acc = [0], 0.0
    for p in parts:
        acc += p
        edges.append(int(round(rows * acc / sum(parts))))
    return edges


def _randn(shape, dtype, gen, scale=1.0):
    t = torch.randn(shape, device="cuda", generator=gen, dtype=DTYPE[dtype])
    return t if scale == 1.0 else t.mul_(scale)


def _tokens(rows, vocab, bits, gen):
    """Tokens as frequent as one over their number, one in forty of them padding (-1)."""
    u = torch.rand(rows, device="cuda", generator=gen, dtype=torch.float64)
    t = (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp(0, vocab - 1)
    return torch.where(torch.rand(rows, device="cuda", generator=gen) < 0.025, -1, t).to(INT[bits])


def _encode(x):
    """Codes [rows, cols] and scales [rows, blocks] of a matrix."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    v = torch.zeros(rows, blocks * BLOCK, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, blocks, BLOCK)
    top = torch.where(v.abs() < math.inf, v.abs(), 0.0).amax(2)
    # the exponent of the largest, one more where it is above 1.75 times its power of two: 448 is 1.75 * 2^8
    e = (((top.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=1)
    q = (v * ((254 - e) << 23).view(torch.float32)[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    q = torch.where((v != 0) & ((q & 127) == 0), q + 1, q)  # what is not 0 is not held as 0
    return q.view(rows, -1)[:, :cols].contiguous().view(torch.float8_e4m3fn), e.to(torch.uint8).view(torch.float8_e8m0fnu)


def _decode(codes, scales):
    e = scales.view(torch.uint8).to(torch.int32)
    return codes.float() * (e << 23).view(torch.float32).repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st, op, way, rows, dtype = {"case": case}, case["op"], case["way"], case["rows"], case["dtype"]
    if case.get("groups"):
        edges = _split(rows, case["groups"], seed)
        st["cap"] = max(b - a for a, b in zip(edges, edges[1:]))
        st["offsets"] = torch.tensor(edges, dtype=torch.int32, device="cuda")
        r, many = random.Random(seed + 1), case.get("matrices") or case.get("tables") or 1
        st["index"] = torch.tensor([r.randrange(many) for _ in range(case["groups"])], dtype=torch.int32, device="cuda")
    if op == "checkpoint":
        st["x"] = _randn((rows, case["fin"]), dtype, gen)
        if way == "encode":
            # the columns of an activation are of different sizes, and some of its values are 0
            size = torch.exp2(torch.randint(-8, 4, (case["fin"],), device="cuda", generator=gen).float())
            st["x"] = torch.where(st["x"] > 1.5, 0.0, st["x"] * size).to(DTYPE[dtype])
        else:
            mats = (case["matrices"],) if case["groups"] else ()
            st["w"] = _randn(mats + (case["fout"], case["fin"]), dtype, gen, case["fin"] ** -0.5)
        if way == "fwd":
            st["b"] = _randn(mats + (case["fout"],), dtype, gen, 0.1)
        if way == "bwd":
            st["dy"] = _randn((rows, case["fout"]), dtype, gen, 0.05)
            st["z"] = _encode(_randn((rows, case["fout"]), dtype, gen))
            if case["keep_x"]:
                st["x"] = _encode(st["x"])
    elif op == "embedding":
        st["tokens"], st["scale"] = _tokens(rows, case["vocab"], case["bits"], gen), case["dim"] ** 0.5
        if way == "fwd":
            st["table"] = _randn(((case["tables"],) if case["groups"] else ()) + (case["vocab"], case["dim"]), dtype, gen, 0.02)
        else:
            st["dy"] = _randn((rows, case["dim"]), dtype, gen, 0.01)
    else:
        z = _randn((rows, case["vocab"]), dtype, gen, 2.5)
        st["tokens"] = _tokens(rows, case["vocab"], case["bits"], gen)
        if case["mask"]:
            z.masked_fill_(torch.rand(case["vocab"], device="cuda", generator=gen) < 0.5, -math.inf)
            if rows > 8:
                z[rows // 3] = -math.inf  # a row that the mask leaves empty
        st["logits"] = z
        if way == "bwd":
            st["dlogp"] = torch.randn(rows, device="cuda", generator=gen).mul_(0.1).sub_(1.0).div_(rows)
            st["dentropy"] = torch.full((rows,), 0.01 / rows, device="cuda")
            st["norm"] = _norm(z.double(), case["scale"]).float()
    if own:
        from paper_2406_05546_amd import dense
        for name in ("x", "z"):
            if isinstance(st.get(name), tuple):
                st[name] = dense.Checkpoint(*st[name])
        if op == "checkpoint" and way == "fwd":
            st["z"] = dense.ps_checkpoint_empty(rows, case["fout"], "cuda:0")
    return st


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _run_own(st):
    from paper_2406_05546_amd import dense, tokens
    case, offsets, index = st["case"], st.get("offsets"), st.get("index")
    op, way = case["op"], case["way"]
    if op == "checkpoint":
        if way == "encode":
            c = dense.ps_checkpoint_encode(st["x"])
            return [c.codes, c.scales]
        if way == "fwd":
            if offsets is None:
                y = dense.ps_linear_forward(st["x"], st["w"], st["b"], activation=case["act"], pre=st["z"])
            else:
                y = dense.ps_grouped_linear_forward(st["x"], offsets, st["w"], st["b"], activation=case["act"], weight_of_group=index, pre=st["z"])
            return [y, st["z"].codes, st["z"].scales]
        if offsets is None:
            return list(dense.ps_linear_backward(st["dy"], st["x"], st["w"], case["act"], pre=st["z"], x_activation=case["x_act"]))
        return list(dense.ps_grouped_linear_backward(st["dy"], st["x"], offsets, st["w"], case["act"], pre=st["z"], weight_of_group=index, x_activation=case["x_act"]))
    if op == "embedding":
        if way == "fwd":
            if offsets is None:
                return tokens.ps_embedding_forward(st["tokens"], st["table"], st["scale"])
            return tokens.ps_grouped_embedding_forward(st["tokens"], offsets, st["table"], st["scale"], table_of_group=index)
        if offsets is None:
            return tokens.ps_embedding_backward(st["dy"], st["tokens"], case["vocab"], st["scale"])
        return tokens.ps_grouped_embedding_backward(st["dy"], st["tokens"], offsets, case["vocab"], st["scale"])
    if way == "fwd":
        p = tokens.ps_logprob_forward(st["logits"], st["tokens"], scale=case["scale"], top=case["top"])
        return [p.logp, p.norm, p.top_logp, p.top_tokens]
    return tokens.ps_logprob_backward(st["logits"], st["tokens"], st["norm"], st["dlogp"], st["dentropy"], scale=case["scale"])


# ---- the plain form -----------------------------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return torch.where(z <= 0, 0.0, z)
    if act == "gelu":
        return 0.5 * z * torch.special.erfc(z * -(0.5 ** 0.5))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return torch.where(z <= 0, 0.0, 1.0)
    if act == "gelu":
        return 0.5 * torch.special.erfc(z * -(0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    s = 1.0 / (1.0 + torch.exp(-z))
    return s * (1.0 + z * (1.0 - s))


def _grouped_places(st):
    row = torch.arange(st["case"]["rows"], device="cuda")
    group = torch.bucketize(row, st["offsets"][1:].long(), right=True)
    return group, row - st["offsets"].long()[group]


def _padded(t, st, group, place):
    out = torch.zeros(st["case"]["groups"], st["cap"], t.shape[1], device="cuda")
    out[group, place] = t.float()
    return out


def _checkpoint_plain(st):
    case, to = st["case"], DTYPE[st["case"]["dtype"]]
    if case["way"] == "encode":
        return list(_encode(st["x"]))
    group, place = _grouped_places(st) if case["groups"] else (None, None)
    w = st["w"].float()
    if case["way"] == "fwd":
        if group is None:
            z = st["x"].float() @ w.t() + st["b"].float()
        else:
            z = torch.bmm(_padded(st["x"], st, group, place), w[st["index"].long()].transpose(1, 2).contiguous())[group, place]
            z = z + st["b"].float()[st["index"].long()[group]]
        return [_act(z, case["act"]).to(to), *_encode(z.to(to))]
    dz = st["dy"].float() * _act_slope(_decode(*st["z"]), case["act"])
    x = _act(_decode(*st["x"]), case["x_act"]) if case["keep_x"] else st["x"].float()
    if group is None:
        return [(dz @ w).to(to), (dz.t() @ x).to(to), dz.sum(0).to(to)]
    pz, px = _padded(dz, st, group, place), _padded(x, st, group, place)
    return [torch.bmm(pz, w[st["index"].long()])[group, place].to(to), torch.bmm(pz.transpose(1, 2).contiguous(), px).to(to), pz.sum(1).to(to)]


def _embedding_plain(st):
    case, t, to = st["case"], st["tokens"].long(), DTYPE[st["case"]["dtype"]]
    there = ((t >= 0) & (t < case["vocab"]))[:, None]
    t = t.clamp(0, case["vocab"] - 1)
    group = _grouped_places(st)[0] if case["groups"] else None
    if case["way"] == "fwd":
        rows = st["table"][t] if group is None else st["table"][st["index"].long()[group], t]
        return torch.where(there, rows.float() * st["scale"], 0.0).to(to)
    dy = torch.where(there, st["dy"].float(), 0.0)
    total = torch.zeros(max(1, case["groups"]) * case["vocab"], case["dim"], device="cuda")
    total.index_add_(0, t if group is None else group * case["vocab"] + t, dy)
    out = (total * st["scale"]).to(to)
    return out if group is None else out.view(case["groups"], case["vocab"], case["dim"])


def _norm(z, scale):
    """Largest logit, logarithm of the sum of exp(scale (z - largest)), entropy.  A row without any has -inf, -inf and 0."""
    m = z.amax(1, keepdim=True)
    u = (z - torch.where(m == -math.inf, 0.0, m)) * scale
    e = torch.exp(u)
    s = e.sum(1, keepdim=True)
    log_s = torch.log(s)
    entropy = torch.where(s > 0, log_s - torch.where(e > 0, e * u, 0.0).sum(1, keepdim=True) / s, 0.0)
    return torch.cat([m, log_s, entropy], 1)


def _logp_of(z, norm, scale):
    """Log probabilities of logits of each row, -inf where the row has none."""
    return torch.where(z == -math.inf, -math.inf, (z - norm[:, :1]) * scale - norm[:, 1:2])


def _logprob_plain(st):
    case, z, t, scale = st["case"], st["logits"].float(), st["tokens"].long(), st["case"]["scale"]
    vocab = case["vocab"]
    there = (t >= 0) & (t < vocab)
    t = t.clamp(0, vocab - 1)[:, None]
    if case["way"] == "fwd":
        norm = _norm(z, scale)
        logp = torch.where(there, _logp_of(z.gather(1, t), norm, scale)[:, 0], 0.0)
        if not case["top"]:
            return [logp, norm, None, None]
        number, left, value, index = torch.arange(vocab, device="cuda"), z.clone(), [], []
        for _ in range(case["top"]):
            best = left.amax(1, keepdim=True)
            at = torch.where(left == best, number, vocab).amin(1, keepdim=True)
            left.scatter_(1, at, -math.inf)
            value.append(best)
            index.append(torch.where(best == -math.inf, -1, at))
        return [logp, norm, _logp_of(torch.cat(value, 1), norm, scale), torch.cat(index, 1).to(torch.int32)]
    logp = _logp_of(z, st["norm"], scale)
    p = torch.exp(logp)
    gl = torch.where(there, st["dlogp"], 0.0)[:, None]
    d = -gl * p - st["dentropy"][:, None] * torch.where(p > 0, p * (logp + st["norm"][:, 2:]), 0.0)
    d.scatter_add_(1, t, gl)
    return torch.where(st["norm"][:, :1] == -math.inf, 0.0, d * scale).to(DTYPE[case["dtype"]])


def run(state):
    if own:
        return _run_own(state)
    return {"checkpoint": _checkpoint_plain, "embedding": _embedding_plain, "logprob": _logprob_plain}[state["case"]["op"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    s, rows, way = {"fp32": 4, "bf16": 2, "fp16": 2}[case["dtype"]], case["rows"], case["way"]
    if case["op"] == "checkpoint":
        fin, held = case["fin"], 1 + 1 / BLOCK
        if way == "encode":
            return {"bytes": rows * fin * (s + held), "flops": 3 * rows * fin}
        fout, mats, groups = case["fout"], min(case["matrices"], case["groups"]) or 1, case["groups"] or 1
        if way == "fwd":
            return {"bytes": s * (rows * (fin + fout) + mats * fout * (fin + 1)) + held * rows * fout, "flops": 2 * rows * fin * fout}
        kept = held * rows * (fout + (fin if case["keep_x"] else 0)) + (0 if case["keep_x"] else s * rows * fin)
        return {"bytes": kept + s * (rows * (fin + fout) + mats * fout * fin + groups * fout * (fin + 1)), "flops": 4 * rows * fin * fout}
    if case["op"] == "embedding":
        dim, token = case["dim"], rows * case["bits"] // 8
        if way == "fwd":
            # a token that comes again is read once
            seen = min(rows, case["vocab"] * max(1, case["tables"]))
            return {"bytes": token + s * dim * (rows + seen), "flops": rows * dim}
        return {"bytes": token + s * dim * (rows + case["vocab"] * max(1, case["groups"])), "flops": rows * dim}
    n = rows * case["vocab"]
    if way == "fwd":
        return {"bytes": s * n + rows * (case["bits"] // 8 + 16 + 8 * case["top"]), "flops": 6 * n}
    return {"bytes": 2 * s * n + rows * (case["bits"] // 8 + 20), "flops": 9 * n}


# ---- the same in 64 bits, from the definitions --------------------------------------------------------------------

def _f64_power(e):
    """2^e, exactly (torch.ldexp takes it from a pow in 32 bits)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _f64_e4m3(x):
    """The nearest e4m3 value, ties to the even one."""
    step = _f64_power(torch.frexp(x).exponent.clamp(min=-5) - 4)  # x is below 2^exponent, or subnormal
    return torch.round(x / step) * step


def _f64_encode(x):
    """Codes and scales as the numbers they stand for."""
    blocks = torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK)).unflatten(1, (-1, BLOCK))
    top = blocks.abs().max(2).values
    # 2^(exponent - 9) times 448 is 0.875 of 2^exponent, which is above the largest, or not
    mantissa, exponent = torch.frexp(top)
    e = (exponent - 9 + (mantissa > 0.875)).clamp(min=-126)
    e = torch.where(top == 0, -126, e)
    scale = _f64_power(e)
    v = blocks / scale[:, :, None]
    q = _f64_e4m3(v)
    q = torch.where((q == 0) & (v != 0), torch.sign(v) * 2.0 ** -9, q)
    return q.flatten(1)[:, :x.shape[1]], scale


def _f64_decode(kept):
    codes, scales = kept if isinstance(kept, tuple) else (kept.codes, kept.scales)
    scale = _f64_power(scales.view(torch.uint8).long() - 127)
    return codes.double() * scale.repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]


def _f64_act(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z)}[act]()


def _f64_slope(z, act):
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return {"relu": lambda: (z > 0).double(), "silu": lambda: torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))}[act]()


def _f64_checkpoint(case, st):
    if case["way"] == "encode":
        return list(_f64_encode(st["x"].double()))
    if case["groups"]:
        edges, index, w = st["offsets"].tolist(), st["index"].tolist(), st["w"]
    else:
        edges, index, w = [0, case["rows"]], [0], st["w"][None]
    parts = [(slice(lo, hi), k) for lo, hi, k in zip(edges, edges[1:], index)]
    if case["way"] == "fwd":
        b = st["b"] if case["groups"] else st["b"][None]
        z = torch.cat([torch.mm(st["x"][s].double(), w[k].double().t()) + b[k].double() for s, k in parts])
        return [_f64_act(z, case["act"]), *_f64_encode(z)]
    dz = st["dy"].double() * _f64_slope(_f64_decode(st["z"]), case["act"])
    x = _f64_act(_f64_decode(st["x"]), case["x_act"]) if case["keep_x"] else st["x"].double()
    dx = torch.cat([torch.mm(dz[s], w[k].double()) for s, k in parts])
    dw = [torch.mm(dz[s].t(), x[s]) for s, _ in parts]
    db = [dz[s].sum(0) for s, _ in parts]
    return [dx, torch.stack(dw), torch.stack(db)] if case["groups"] else [dx, dw[0], db[0]]


def _f64_embedding(case, st):
    tokens, vocab = st["tokens"].long(), case["vocab"]
    kept = (tokens >= 0) & (tokens < vocab)
    owner = torch.zeros_like(tokens)
    if case["groups"]:
        sizes = (st["offsets"][1:] - st["offsets"][:-1]).long()
        owner = torch.repeat_interleave(torch.arange(case["groups"], device="cuda"), sizes)
    if case["way"] == "fwd":
        out = torch.zeros(case["rows"], case["dim"], dtype=torch.float64, device="cuda")
        at = (st["index"].long()[owner[kept]], tokens[kept]) if case["groups"] else tokens[kept]
        out[kept] = st["table"][at].double() * st["scale"]
        return out
    out = torch.zeros(max(1, case["groups"]), vocab, case["dim"], dtype=torch.float64, device="cuda")
    out.index_put_((owner[kept], tokens[kept]), st["dy"][kept].double() * st["scale"], accumulate=True)
    return out if case["groups"] else out[0]


def _f64_logprob(case, st):
    scale, vocab, tokens = case["scale"], case["vocab"], st["tokens"].long()
    rows = torch.arange(case["rows"], device="cuda")
    empty = torch.isneginf(st["logits"]).all(1)
    kept = (tokens >= 0) & (tokens < vocab)
    given = torch.where(kept, tokens, 0)
    if case["way"] == "bwd":
        out = []
        for lo in range(0, case["rows"], 1024):
            s = slice(lo, lo + 1024)
            logp = torch.log_softmax(st["logits"][s].double() * scale, 1)
            p = torch.exp(logp)
            plogp = torch.xlogy(p, p)
            entropy = -plogp.sum(1, keepdim=True)
            gl = (st["dlogp"][s].double() * kept[s])[:, None]
            d = -(gl * p) - st["dentropy"][s].double()[:, None] * (plogp + p * entropy)
            d[rows[s] - lo, given[s]] += gl[:, 0]
            d[empty[s]] = 0.0
            out.append(d * scale)
        return torch.cat(out)
    found = []
    for lo in range(0, case["rows"], 1024):
        s = slice(lo, lo + 1024)
        z = st["logits"][s].double()
        logp = torch.log_softmax(z * scale, 1)
        p = torch.exp(logp)
        largest = z.max(1).values
        log_s = torch.logsumexp(z * scale, 1) - largest * scale
        one = logp[rows[s] - lo, given[s]]
        entropy = -torch.xlogy(p, p).sum(1)
        one = torch.where(kept[s], torch.where(empty[s], -math.inf, one), 0.0)
        norm = torch.stack([largest, torch.where(empty[s], -math.inf, log_s), torch.where(empty[s], 0.0, entropy)], 1)
        top = logp.topk(min(case["top"], vocab), 1).values if case["top"] else None
        if top is not None:
            top = torch.where(empty[s][:, None], -math.inf, torch.nn.functional.pad(top, (0, case["top"] - top.shape[1]), value=-math.inf))
        found.append((one, norm, top))
    return [torch.cat([f[0] for f in found]), torch.cat([f[1] for f in found]), torch.cat([f[2] for f in found]) if case["top"] else None, None]


def exact(case, seed):
    st = prepare(case, seed)
    return {"checkpoint": _f64_checkpoint, "embedding": _f64_embedding, "logprob": _f64_logprob}[case["op"]](case, st)
