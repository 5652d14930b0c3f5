"""Operators that explain a token model's answer, as measured cases.

The players are prompt tokens.  New tokens' keys and values enter a paged cache
(`append`); every coalition's new token attends over the one cached prompt,
seeing the positions its mask keeps, and over tokens of its own (`attend`);
the answer's log probability, with entropy, rank and alternatives, is the
coalition's value (`logprobs`), and its gradient by the logits serves gradient
attributions (`gradient`).

Where `own` is false, `run` computes each operator from elementary torch
operations in 32 bits, rounded once at the end; where it is true it calls the
framework.  Both take what `prepare` gives.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _attend(name, dtype, heads, kv_heads, dim, page, rows, shared, groups, own_max, players, first):
    return dict(name=name, kind="attend", dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, page=page, rows=rows,
                shared=shared, groups=groups, own_max=own_max, players=players, first=first)


def listed():
    return [
        # one token of one sequence enters the cache: an interactive decode step, where latency counts
        dict(name="append one", kind="append", dtype="bf16", heads=32, kv_heads=8, dim=128, rot=128, page=64, tokens=1,
             seqs=1, history=1000, interleaved=False),
        # prompts enter the cache: 20,000 tokens of four sequences
        dict(name="append prompts", kind="append", dtype="bf16", heads=32, kv_heads=8, dim=128, rot=128, page=64,
             tokens=20000, seqs=4, history=1000, interleaved=False),
        # one sequence's new token over its cache: an interactive decode step
        _attend("attend one", "bf16", 32, 8, 128, 64, rows=1, shared=0, groups=0, own_max=4000, players=0, first=0),
        # a batch of sequences of very unlike lengths, one to 20,000 tokens, on short pages
        _attend("attend ragged", "f16", 32, 8, 128, 16, rows=64, shared=0, groups=0, own_max=20000, players=0, first=0),
        # 2,000 coalitions of a short prompt's 59 tokens, a 32-bit model
        _attend("attend coalitions 32 bits", "f32", 8, 8, 64, 64, rows=2000, shared=59, groups=1, own_max=3, players=59,
                first=0),
        # 10,000 coalitions of 400 prompt tokens behind a 17-token instruction that every coalition keeps
        _attend("attend coalitions", "bf16", 32, 8, 128, 16, rows=10000, shared=417, groups=1, own_max=4, players=400,
                first=17),
        # a long prompt, with the empty and the full coalition beside 2,000 others
        _attend("attend coalitions long", "bf16", 32, 8, 128, 64, rows=2002, shared=3851, groups=1, own_max=1,
                players=3851, first=0),
        # the next token of one sequence, with 20 alternatives
        dict(name="logprobs one", kind="logprobs", dtype="bf16", rows=1, vocab=131072, top=20),
        # the answer token under 10,000 coalitions
        dict(name="logprobs coalitions", kind="logprobs", dtype="bf16", rows=10000, vocab=32768, top=5),
        # the classes of a node classifier under 100,000 coalitions
        dict(name="logprobs classes", kind="logprobs", dtype="f32", rows=100000, vocab=41, top=3),
        # gradients by the logits of a batch, with a vocabulary of odd size
        dict(name="gradient", kind="gradient", dtype="bf16", rows=2000, vocab=50021),
        # gradients of a few answers in 32 bits
        dict(name="gradient few", kind="gradient", dtype="f32", rows=16, vocab=32768),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "coalitions", "coalitions", "logprobs", "logprobs", "gradient"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    if kind in ("logprobs", "gradient"):
        rows = _log(rng, 1, 25000)
        vocab = _log(rng, 2, min(131072, (320 if kind == "logprobs" else 100) * 10**6 // rows))
        if kind == "gradient":
            return dict(kind=kind, dtype=dtype, rows=rows, vocab=vocab)
        return dict(kind=kind, dtype=dtype, rows=rows, vocab=vocab, top=min(vocab, rng.choice([0, 1, 5, 20])))
    kv_heads, share = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 7, 8])
    dim, page = rng.choice([64, 80, 128, 128, 256]), rng.choice([16, 24, 32, 64, 128])
    heads = min(kv_heads * share, 32 // kv_heads * kv_heads)
    if kind == "append":
        # prompts and steps of up to 64 sequences, or one step of many coalitions
        many = rng.random() < 0.3
        tokens = _log(rng, 100, 10000) if many else _log(rng, 1, 20000)
        return dict(kind=kind, dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, tokens=tokens,
                    page=min(page, 32) if many else page, seqs=tokens if many else _log(rng, 1, min(tokens, 64)),
                    history=8 if many else 1000, rot=rng.choice([dim, dim, dim // 2]),
                    interleaved=rng.random() < 0.5)
    if kind == "decode":
        rows = _log(rng, 1, 100)
        return dict(kind="attend", dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, page=page, rows=rows,
                    shared=0, groups=0, own_max=_log(rng, 1, min(30000, 10**9 // (rows * kv_heads * dim))), players=0,
                    first=0)
    groups = rng.choice([1, 1, 2, 3])
    rows = groups * _log(rng, 10, 10000 // groups)
    shared = _log(rng, 16, min(4000, 16 * 10**9 // (rows * heads * dim)))
    first = rng.choice([0, rng.randrange(shared)])
    return dict(kind="attend", dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, page=page, rows=rows,
                shared=shared, groups=groups, own_max=_log(rng, 1, 8), players=shared - first, first=first)


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    return dict(case=case, **{"append": _prepare_append, "attend": _prepare_attend, "logprobs": _prepare_logits,
                              "gradient": _prepare_logits}[case["kind"]](case, gen))


def _normal(gen, *size):
    return torch.randn(size, device=DEV, generator=gen)


def _pages(gen, rows, length, page, taken=0):
    """A page table of `rows` sequences of up to `length` tokens, pages in no order, behind `taken` other pages."""
    per = max(1, -(-length // page))
    return (taken + torch.randperm(rows * per, device=DEV, generator=gen)).view(rows, per).to(torch.int32)


def _spread(gen, rows, lo, hi):
    """`rows` lengths from hi down to lo, evenly in the logarithm (from 0: evenly), in random order."""
    at = torch.linspace(0, 1, rows, device=DEV, dtype=torch.float64)
    x = hi * (1 - at) if lo == 0 else hi * (lo / hi) ** at
    return x.round().to(torch.int32)[torch.randperm(rows, device=DEV, generator=gen)]


def _prepare_append(case, gen):
    n, seqs, dim, page = case["tokens"], case["seqs"], case["dim"], case["page"]
    dtype = TYPES[case["dtype"]]
    # a model's projection holds queries, keys and values side by side
    qkv = _normal(gen, n, case["heads"] + 2 * case["kv_heads"], dim).to(dtype)
    per = -(-n // seqs)                                     # tokens of a sequence, the last ones fewer
    start = torch.randint(0, case["history"], (seqs,), device=DEV, generator=gen)  # what the cache holds of it already
    at = torch.arange(n, device=DEV)
    rows = at // per
    index = start[rows] + at % per
    table = _pages(gen, seqs, case["history"] + per, page)
    angle = torch.arange(case["history"] + per, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, case["rot"], 2, device=DEV, dtype=torch.float64) / case["rot"])
    cache = torch.zeros((2, table.numel(), page, case["kv_heads"], dim), dtype=dtype, device=DEV)
    return dict(qkv=qkv, rows=rows.to(torch.int32), index=index.to(torch.int32), table=table, k_pages=cache[0],
                v_pages=cache[1], cos=angle.cos().float(), sin=angle.sin().float())


def _prepare_attend(case, gen):
    rows, groups, page, dim = case["rows"], case["groups"], case["page"], case["dim"]
    dtype = TYPES[case["dtype"]]
    q = (1.5 * _normal(gen, rows, case["heads"], dim)).to(dtype)
    table = _pages(gen, rows, case["own_max"], page)
    # sequences of one to own_max tokens; coalitions have none to own_max tokens of their own
    lengths = _spread(gen, rows, 0 if groups and case["own_max"] > 1 else 1, case["own_max"])
    used, state = table.numel(), {}
    if groups:
        shared = _pages(gen, groups, case["shared"], page, used)
        used += shared.numel()
        # coalitions of every size in pairs of complements, the last pair the empty and the full one
        m, half = case["players"], -(-rows // 2)
        keep = torch.rand((half, m), device=DEV, generator=gen) < torch.rand((half, 1), device=DEV, generator=gen)
        keep[-1] = False
        keep = torch.cat([keep, ~keep])[:rows]
        bits = torch.zeros((rows, -(-m // 64) * 64), dtype=torch.int64, device=DEV)
        bits[:, :m] = keep
        state = dict(masks=(bits.view(rows, -1, 64) << torch.arange(64, device=DEV)).sum(2), shared_table=shared,
                     shared_lengths=torch.full((groups,), case["shared"], dtype=torch.int32, device=DEV))
    k = torch.empty((used, page, case["kv_heads"], dim), dtype=dtype, device=DEV).normal_(generator=gen)
    v = torch.empty_like(k).normal_(generator=gen)
    return dict(q=q, k_pages=k, v_pages=v, table=table, lengths=lengths, **state)


def _prepare_logits(case, gen):
    rows, vocab = case["rows"], case["vocab"]
    x = 2.5 * _normal(gen, rows, vocab)
    # an answer is mostly among the likely tokens; every 16th row forbids some tokens
    targets = torch.randint(0, vocab, (rows,), device=DEV, generator=gen)
    x[torch.arange(rows, device=DEV), targets] += 6 * torch.rand(rows, device=DEV, generator=gen)
    banned = torch.rand((x[::16].shape[0], vocab), device=DEV, generator=gen) < 0.05
    banned[:, 0] = False
    x[::16] = x[::16].masked_fill(banned, -math.inf)
    state = dict(logits=x.to(TYPES[case["dtype"]]), targets=targets)
    if case["kind"] == "gradient":                          # what the forward pass left
        del x, banned
        y = state["logits"].float()
        lse = torch.logsumexp(y, 1)
        state |= dict(lse=lse, entropy=lse - (torch.exp(y - lse[:, None]) * y.nan_to_num(neginf=0.0)).sum(1),
                      grad_logprob=_normal(gen, rows), grad_entropy=0.1 * _normal(gen, rows))
    return state


def run(state):
    kind = state["case"]["kind"]
    return {"append": _append, "attend": _attention, "logprobs": _logprobs, "gradient": _gradient}[kind](state)


def _append(s):
    case = s["case"]
    q, k, v = s["qkv"].split([case["heads"], case["kv_heads"], case["kv_heads"]], dim=1)
    if own:
        from paper_2401_04829_amd import answers
        cache = answers.PagedCache(s["k_pages"], s["v_pages"])
        q = answers.append_tokens(cache, k, v, s["table"], s["index"], rows=s["rows"], q=q, cos=s["cos"], sin=s["sin"],
                                  interleaved=case["interleaved"])
        return q, s["k_pages"], s["v_pages"]
    index = s["index"].long()
    page = s["table"][s["rows"].long(), index // case["page"]].long()
    s["k_pages"][page, index % case["page"]] = _rotate(k, s["cos"][index], s["sin"][index], case)
    s["v_pages"][page, index % case["page"]] = v
    return _rotate(q, s["cos"][index], s["sin"][index], case), s["k_pages"], s["v_pages"]


def _rotate(x, cos, sin, case):
    rot = case["rot"]
    y, c, s = x.float(), cos[:, None], sin[:, None]
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if case["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _attention(s):
    case = s["case"]
    scale = 1 / math.sqrt(case["dim"])
    if own:
        from paper_2401_04829_amd import answers
        cache = answers.PagedCache(s["k_pages"], s["v_pages"])
        return answers.attend(cache, s["q"], table=s["table"], lengths=s["lengths"], max_length=case["own_max"],
                              shared_table=s.get("shared_table"), shared_lengths=s.get("shared_lengths"),
                              max_shared=case["shared"], masks=s.get("masks"), num_players=case["players"],
                              first_player=case["first"], scale=scale, return_lse=True)
    rows, heads, kv, dim = case["rows"], case["heads"], case["kv_heads"], case["dim"]
    q = s["q"].float().view(rows, kv, heads // kv, dim)
    k, v = _gather(s, s["table"], case["own_max"])
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale             # [rows, kv, heads / kv, own]
    seen = torch.arange(case["own_max"], device=DEV) < s["lengths"][:, None]
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    if not case["groups"]:
        p, lse = _softmax(x)
        return torch.matmul(p, v).view(rows, heads, dim).to(s["q"].dtype), lse.view(rows, heads)
    g, r = case["groups"], rows // case["groups"]
    sk, sv = _gather(s, s["shared_table"], case["shared"])
    shared_q = q.view(g, r, kv, heads // kv, dim).transpose(1, 2).reshape(g, kv, -1, dim)
    sx = (torch.matmul(shared_q, sk.transpose(2, 3).contiguous()) * scale).view(g, kv, r, heads // kv, -1)
    sx = sx.transpose(1, 2).reshape(rows, kv, heads // kv, -1)              # [rows, kv, heads / kv, shared]
    keep = (s["masks"][:, :, None] >> torch.arange(64, device=DEV) & 1).bool().flatten(1)[:, :case["players"]]
    seen = torch.ones((rows, case["shared"]), dtype=torch.bool, device=DEV)
    seen[:, case["first"]:case["first"] + case["players"]] = keep
    sx = sx.masked_fill(~seen[:, None, None], -math.inf)
    p, lse = _softmax(torch.cat([sx, x], -1))
    sp = p[..., :case["shared"]].view(g, r, kv, heads // kv, -1).transpose(1, 2).reshape(g, kv, -1, case["shared"])
    out = torch.matmul(sp, sv).view(g, kv, r, heads // kv, dim).transpose(1, 2).reshape(rows, kv, heads // kv, dim)
    out = out + torch.matmul(p[..., case["shared"]:], v)
    return out.reshape(rows, heads, dim).to(s["q"].dtype), lse.reshape(rows, heads)


def _gather(s, table, length):
    """Keys and values of the table's sequences in 32 bits, [rows, kv heads, length, dim]."""
    pick = [x[table.long()].flatten(1, 2)[:, :length].float().transpose(1, 2).contiguous()
            for x in (s["k_pages"], s["v_pages"])]
    return pick[0], pick[1]


def _softmax(x):
    """Softmax and log sum of exponentials over the last axis; a row with nothing in it gives 0 and -inf."""
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top.masked_fill(top == -math.inf, 0.0))
    total = e.sum(-1, keepdim=True)
    return e / total.masked_fill(total == 0, 1.0), (top + torch.log(total)).squeeze(-1)


def _logprobs(s):
    x, targets, top = s["logits"], s["targets"], s["case"]["top"]
    if own:
        from paper_2401_04829_amd import answers
        r = answers.token_logprobs(x, targets, top=top)
        return r.logprob, r.entropy, r.lse, r.rank, r.top_logprob, r.top_id
    y = x.float()
    most = y.amax(1, keepdim=True)
    e = torch.exp(y - most)
    total = e.sum(1, keepdim=True)
    lse = (most + torch.log(total))[:, 0]
    # p log p with p = e / total; nothing where p is 0
    entropy = torch.log(total)[:, 0] - (e * (y - most).masked_fill(e == 0, 0.0)).sum(1) / total[:, 0]
    chosen = y.gather(1, targets[:, None])
    rank = (y > chosen).sum(1).to(torch.int32)
    # one whole number for each logit, in the logits' order and among equal ones the lowest place first
    bits = (y + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32
    where = (order - torch.arange(y.shape[1], device=DEV)).topk(top, 1).indices
    return chosen[:, 0] - lse, entropy, lse, rank, y.gather(1, where) - lse[:, None], where.to(torch.int32)


def _gradient(s):
    x, targets = s["logits"], s["targets"]
    if own:
        from paper_2401_04829_amd import answers
        return answers.token_logprobs_backward(x, targets, s["lse"], s["entropy"], s["grad_logprob"],
                                               s["grad_entropy"])
    logp = x.float() - s["lse"][:, None]
    p = torch.exp(logp)
    d = -p * (s["grad_logprob"][:, None]
              + s["grad_entropy"][:, None] * (logp.masked_fill(p == 0, 0.0) + s["entropy"][:, None]))
    d[torch.arange(x.shape[0], device=DEV), targets] += s["grad_logprob"]
    return d.to(x.dtype)


def work(case):
    b, kind = BYTES[case["dtype"]], case["kind"]
    if kind == "append":
        n, width = case["tokens"], (case["heads"] + 2 * case["kv_heads"]) * case["dim"]
        # each token's vectors in and out, its angles, its place
        return {"bytes": n * (2 * width * b + 4 * case["rot"] + 12),
                "flops": 3 * n * (case["heads"] + case["kv_heads"]) * case["rot"]}
    if kind == "attend":
        rows, heads, dim, hi = case["rows"], case["heads"], case["dim"], case["own_max"]
        if case["groups"]:
            own_keys = rows * (hi / 2 if hi > 1 else 1)
        else:
            own_keys = rows * ((hi - 1) / math.log(hi) if rows > 1 and hi > 1 else hi)
        # half of the (coalition, player) pairs are kept
        pairs = own_keys + rows * (case["shared"] - case["players"] / 2)
        keys = own_keys + case["groups"] * case["shared"]
        return {"bytes": int(2 * keys * case["kv_heads"] * dim * b + 2 * rows * heads * dim * b + 4 * rows * heads
                             + rows * case["players"] / 8 + 4 * keys / case["page"] + 4 * rows),
                "flops": int(4 * pairs * heads * dim)}
    n = case["rows"] * case["vocab"]
    if kind == "gradient":
        return {"bytes": 2 * n * b + 24 * case["rows"], "flops": 6 * n}
    return {"bytes": n * b + case["rows"] * (24 + 8 * case["top"]), "flops": 6 * n}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "logprobs": _exact_logprobs,
            "gradient": _exact_gradient}[case["kind"]](case, s)


def _exact_append(case, s):
    heads, kv, rot, page = case["heads"], case["kv_heads"], case["rot"], case["page"]
    n, dim = case["tokens"], case["dim"]
    at = torch.arange(rot // 2, device=DEV)
    first, second = (2 * at, 2 * at + 1) if case["interleaved"] else (at, at + rot // 2)
    # as complex numbers, turned by cos + i sin
    turn = torch.complex(s["cos"].double(), s["sin"].double())[s["index"].long()][:, None]
    x = s["qkv"].double()
    z = torch.complex(x[:, :heads + kv, first], x[:, :heads + kv, second]) * turn
    x[:, :heads + kv, first], x[:, :heads + kv, second] = z.real, z.imag
    slot = s["table"].long()[s["rows"].long(), s["index"].long() // page] * page + s["index"].long() % page
    shape = s["k_pages"].shape
    out = torch.zeros((2, shape[0] * page, kv, dim), dtype=torch.float64, device=DEV)
    out[0].index_copy_(0, slot, x[:, heads:heads + kv])
    out[1].index_copy_(0, slot, x[:, heads + kv:])
    return x[:n, :heads], out[0].view(shape), out[1].view(shape)


def _exact_attend(case, s):
    rows, heads, dim, page = case["rows"], case["heads"], case["dim"], case["page"]
    per, share = max(1, rows // max(1, case["groups"])), heads // case["kv_heads"]
    out = torch.zeros((rows, heads, dim), dtype=torch.float64, device=DEV)
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device=DEV)
    q = s["q"].double() / math.sqrt(dim)
    if case["groups"]:
        width = case["players"]
        word, bit = torch.arange(width, device=DEV) // 64, torch.arange(width, device=DEV) % 64
        absent = (s["masks"][:, word] >> bit) % 2 == 0
        own_at = torch.arange(case["own_max"], device=DEV)
        place = s["table"].long()[:, own_at // page] * page + own_at % page             # [rows, own_max]
        late = own_at >= s["lengths"][:, None]
        at = torch.arange(case["shared"], device=DEV)
        first, last = case["first"], case["first"] + width
        for g in range(case["groups"]):
            r = slice(g * per, (g + 1) * per)
            common = s["shared_table"].long()[g, at // page] * page + at % page
            for h in range(heads):
                k = s["k_pages"][:, :, h // share].reshape(-1, dim)
                v = s["v_pages"][:, :, h // share].reshape(-1, dim)
                x = q[r, h] @ k[common].double().T
                x[:, first:last][absent[r]] = -math.inf
                y = (q[r, h][:, None] * k[place[r]].double()).sum(2)
                y[late[r]] = -math.inf
                total = torch.logsumexp(torch.cat([x, y], 1), 1)
                lse[r, h] = total
                total = torch.where(total == -math.inf, torch.zeros_like(total), total)[:, None]
                out[r, h] = torch.exp(x - total) @ v[common].double() + (
                    torch.exp(y - total)[:, :, None] * v[place[r]].double()).sum(1)
        return out, lse
    length = s["lengths"].tolist()
    for b in range(rows):
        at = torch.arange(length[b], device=DEV)
        place = s["table"].long()[b, at // page]
        for h in range(case["kv_heads"]):
            k, v = (x[place, at % page, h].double() for x in (s["k_pages"], s["v_pages"]))
            x = q[b, h * share:(h + 1) * share] @ k.T
            lse[b, h * share:(h + 1) * share] = torch.logsumexp(x, 1)
            out[b, h * share:(h + 1) * share] = torch.softmax(x, 1) @ v
    return out, lse


def _exact_logprobs(case, s):
    rows, top = case["rows"], case["top"]
    lp, ent, lse = (torch.empty(rows, dtype=torch.float64, device=DEV) for _ in range(3))
    best = torch.empty((rows, top), dtype=torch.float64, device=DEV)
    step = max(1, 2**27 // case["vocab"])
    for r in range(0, rows, step):
        x = s["logits"][r:r + step].double()
        logp = torch.log_softmax(x, 1)
        lp[r:r + step] = logp.gather(1, s["targets"][r:r + step, None])[:, 0]
        lse[r:r + step] = torch.logsumexp(x, 1)
        ent[r:r + step] = torch.special.entr(logp.exp()).sum(1)
        best[r:r + step] = logp.topk(top, 1).values
    # ranks and places are whole numbers, which the plain form has exactly
    return lp, ent, lse, None, best, None


def _exact_gradient(case, s):
    x = s["logits"].double()
    logp = x - s["lse"].double()[:, None]
    hot = torch.zeros_like(x).scatter_(1, s["targets"][:, None], 1.0)
    ent = torch.special.entr(logp.exp()) - logp.exp() * s["entropy"].double()[:, None]     # -p (log p + H)
    return s["grad_logprob"].double()[:, None] * (hot - logp.exp()) + s["grad_entropy"].double()[:, None] * ent
