"""The operators of a step of drafted tokens as cases that can be timed and checked, each in two forms.

  groups   a linear layer whose 4-bit weights have a step size per group of input channels; its input stays as it is
  rotate   queries and keys between that layer and the cache: a norm per head and the rotation by position
  tree     attention of a tree of drafted tokens over the paged 8-bit cache: a token sees what the sequence held before
           and, of the drafted ones, those that its bits name
  scores   what the model makes of the drafted tokens: log probabilities of given tokens, the entropy of each
           distribution and its most probable alternatives

With `own` false a case runs in its plain form, elementary torch operations; with `own` true through
`paper_2302_01382_amd.mpq`.

Weights: codes in -8..7 as two's-complement nibbles [n, k / 2], the even channel in the low half; steps [n, k / group].
The cache: key codes int8 [pages, heads, page, dim], value codes int8 [pages, heads, page / 4, dim, 4] (four tokens of a
channel side by side), maxima float32 [pages, heads] of either, value = code * maximum / (2^(bits-1) - 1).  Position p of
sequence s is on page table[s, p // page].  Bit j of row i's bits (int64 words of 64): row i sees its sequence's drafted
token j.
"""
import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-6


def listed():
    return [
        # one token through a square layer of BERT-large's width: latency is all there is to it
        {"name": "groups_one_token", "kind": "groups", "m": 1, "k": 1024, "n": 1024, "group": 64, "type": "bf16", "steps": "fp32", "act": "none"},
        # one token through a wide layer: the weights' bytes count
        {"name": "groups_one_token_wide", "kind": "groups", "m": 1, "k": 4096, "n": 12288, "group": 128, "type": "fp16", "steps": "fp16", "act": "none"},
        # the drafted tokens of a few sequences through a feed-forward layer, the finest groups
        {"name": "groups_drafted", "kind": "groups", "m": 61, "k": 4096, "n": 11008, "group": 32, "type": "bf16", "steps": "bf16", "act": "gelu"},
        # one token's heads, BERT-large's, in 32 bits: latency
        {"name": "rotate_one_token", "kind": "rotate", "rows": 1, "q_heads": 16, "heads": 16, "dim": 64, "rot": 64, "pairs": False, "far": 512, "type": "fp32"},
        # drafted tokens of a serving batch, far into their sequences
        {"name": "rotate_drafted", "kind": "rotate", "rows": 997, "q_heads": 32, "heads": 8, "dim": 128, "rot": 128, "pairs": False, "far": 1000000, "type": "bf16"},
        # prompts, half of each head rotated, in neighbouring pairs
        {"name": "rotate_prompts", "kind": "rotate", "rows": 12289, "q_heads": 32, "heads": 8, "dim": 128, "rot": 64, "pairs": True, "far": 20000, "type": "fp16"},
        # five drafted tokens of one sequence of the length BERT's inputs have: latency
        {"name": "tree_one_short", "kind": "tree", "seqs": 1, "new": 5, "held": 383, "q_heads": 16, "heads": 16, "dim": 64, "page": 16, "type": "fp32", "bits": 8},
        # a serving batch with a small tree each, four query heads to a key head, ragged lengths
        {"name": "tree_batch", "kind": "tree", "seqs": 24, "new": 13, "held": 8000, "q_heads": 32, "heads": 8, "dim": 128, "page": 64, "type": "bf16", "bits": 8},
        # a wide tree behind one very long sequence: work has to be split along it
        {"name": "tree_one_long", "kind": "tree", "seqs": 1, "new": 61, "held": 65500, "q_heads": 32, "heads": 8, "dim": 128, "page": 128, "type": "fp16", "bits": 8},
        # one token's scores
        {"name": "scores_one", "kind": "scores", "rows": 1, "vocab": 32768, "top": 5, "hidden": 0.0, "type": "bf16"},
        # the scores of drafted tokens, an odd vocabulary of which a part is ruled out, logits in 32 bits
        {"name": "scores_drafted", "kind": "scores", "rows": 190, "vocab": 100003, "top": 20, "hidden": 0.02, "type": "fp32"},
        # a prompt's scores
        {"name": "scores_prompt", "kind": "scores", "rows": 2500, "vocab": 65536, "top": 8, "hidden": 0.0, "type": "bf16"},
    ]


def _log(rng, low, high):
    """A whole number, spread over the logarithm of the range."""
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    kind = rng.choice(["groups", "rotate", "tree", "scores"])
    t = rng.choice(["fp32", "bf16", "fp16"])
    if kind == "groups":
        m, n, group = _log(rng, 1, 64), _log(rng, 64, 12288), rng.choice([32, 64, 128])
        k = max(1, _log(rng, 128, 8192) // group) * group
        if rng.random() < 0.6:  # layers mostly have round sizes
            n = n // 64 * 64
        while m * k * n > 61 * 4096 * 11008 or k * n > 4096 * 12288:
            n = n // 2
        return {"kind": kind, "m": m, "k": k, "n": n, "group": group, "type": t, "steps": rng.choice(["fp32", "fp32", "bf16", "fp16"]),
                "act": rng.choice(["none", "none", "relu", "gelu"])}
    if kind == "rotate":
        heads, dim = rng.choice([1, 2, 4, 8, 12]), rng.choice([64, 80, 96, 128, 256])
        q_heads, rows = heads * rng.choice([1, 2, 4, 7, 8]), _log(rng, 1, 12289)
        while rows * (q_heads + heads) * dim * SIZE[t] > 12289 * 40 * 128 * 2:
            rows = rows // 2
        return {"kind": kind, "rows": rows, "q_heads": q_heads, "heads": heads, "dim": dim, "rot": rng.choice([dim, dim, dim // 2]),
                "pairs": rng.random() < 0.4, "far": _log(rng, 64, 1000000), "type": t}
    if kind == "tree":
        heads, group, dim = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 2, 4, 7, 8]), rng.choice([64, 80, 96, 128, 256])
        seqs, new, held = _log(rng, 1, 32), _log(rng, 1, 100), _log(rng, 1, 65536)
        while seqs * (new + held) * heads * dim > 24 * 8013 * 8 * 128 or seqs * new * (new + held) * heads * group * dim > 61 * 65561 * 32 * 128:
            held = held // 2
        return {"kind": kind, "seqs": seqs, "new": new, "held": held, "q_heads": heads * group, "heads": heads, "dim": dim,
                "page": rng.choice([16, 32, 64, 128]), "type": t, "bits": rng.choice([8, 8, 6, 4])}
    rows, vocab = _log(rng, 1, 4096), _log(rng, 1000, 160000)
    if rng.random() < 0.5:
        vocab = max(1, vocab // 64) * 64
    while rows * vocab * SIZE[t] > 2500 * 65536 * 2:
        rows = rows // 2
    return {"kind": kind, "rows": rows, "vocab": vocab, "top": rng.choice([1, 5, 8, 20, 32]), "hidden": rng.choice([0.0, 0.0, 0.02, 0.5]), "type": t}


def _lengths(case):
    """(new, held) tokens of each sequence: the case's numbers are the largest, its batch is ragged."""
    rng = random.Random("%(seqs)d %(new)d %(held)d %(heads)d" % case)
    new = [case["new"]] + [rng.randint((case["new"] + 1) // 2, case["new"]) for _ in range(case["seqs"] - 1)]
    held = [case["held"]] + [rng.randint(case["held"] // 2, case["held"]) for _ in range(case["seqs"] - 1)]
    return new, held


def _trees(case, new, seed):
    """Bits of every row as Python integers: itself and its ancestors.  Each drafted token continues one of the eight
    before it, or the sequence itself."""
    rng, rows = random.Random(seed), []
    for n in new:
        seen = []
        for i in range(n):
            parent = rng.randint(max(-1, i - 8), i - 1)
            seen.append(1 << i | (seen[parent] if parent >= 0 else 0))
        rows += seen
    return rows


def _codes(shape, bits, g):
    """Codes as a bell-shaped tensor leaves them on the grid of its own maximum."""
    q = 2 ** (bits - 1) - 1
    return torch.randn(shape, device="cuda", generator=g).mul_(q / 3.5).round_().clamp_(-q, q).to(torch.int8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s, t = dict(case), TYPES[case["type"]]
    if case["kind"] == "groups":
        m, k, n = case["m"], case["k"], case["n"]
        c = _codes((n, k), 4, g).view(n, k // 2, 2).to(torch.int16) & 15
        s["w"] = (c[..., 0] | c[..., 1] << 4).to(torch.uint8)
        s["w_step"] = ((torch.rand(n, k // case["group"], device="cuda", generator=g) + 0.5) * 0.01).to(TYPES[case["steps"]])
        x = torch.randn(m, k, device="cuda", generator=g)
        x[:, torch.randint(0, k, (6,), device="cuda", generator=g)] *= 20  # a few channels are always much larger
        s["x"] = x.to(t)
        return s
    if case["kind"] == "rotate":
        rows, q_heads, heads, dim, rot = (case[n] for n in ("rows", "q_heads", "heads", "dim", "rot"))
        # queries, keys and values lie in one tensor, as the layer that makes them leaves them
        width = torch.exp(torch.randn(q_heads + 2 * heads, 1, device="cuda", generator=g))
        qkv = (torch.randn(rows, q_heads + 2 * heads, dim, device="cuda", generator=g) * width).to(t)
        s["q"], s["k"] = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads]
        s["q_weight"], s["k_weight"] = (1 + 0.2 * torch.randn(dim, device="cuda", generator=g) for _ in range(2))
        s["positions"] = torch.randint(0, case["far"], (rows,), device="cuda", generator=g).to(torch.int32)
        s["frequencies"] = (10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)).float()
        return s
    if case["kind"] == "tree":
        new, held = _lengths(case)
        heads, dim, page = case["heads"], case["dim"], case["page"]
        long = max(a + b for a, b in zip(new, held))
        per_seq = -(-long // page)
        pages = case["seqs"] * per_seq + 3
        s["table"] = torch.randperm(pages, device="cuda", generator=g)[: case["seqs"] * per_seq].view(case["seqs"], per_seq).to(torch.int32)
        s["k_codes"], s["v_codes"] = _codes((pages, heads, page, dim), case["bits"], g), _codes((pages, heads, page // 4, dim, 4), case["bits"], g)
        s["k_absmax"], s["v_absmax"] = ((torch.rand(pages, heads, device="cuda", generator=g) + 1) * 2.5 for _ in range(2))
        s["kv_len"] = torch.tensor([a + b for a, b in zip(new, held)], dtype=torch.int32, device="cuda")
        starts = [sum(new[:i]) for i in range(len(new) + 1)]
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["rows"], s["max_new"], s["max_len"] = sum(new), max(new), long
        s["q"] = torch.randn(s["rows"], case["q_heads"], dim, device="cuda", generator=g).to(t)
        words = (max(new) + 63) // 64
        bits = [[(b >> 64 * w & (1 << 64) - 1) - (b >> 64 * w + 63 & 1) * (1 << 64) for w in range(words)] for b in _trees(case, new, seed)]
        s["tree"] = torch.tensor(bits, dtype=torch.int64, device="cuda")
        if own:  # the handles that a serving program keeps from call to call: the tensors above and their sizes, nothing computed
            from paper_2302_01382_amd import mpq

            s["cache"] = mpq.KvCache(s["k_codes"], s["v_codes"], s["k_absmax"], s["v_absmax"], case["bits"])
            s["batch"] = mpq.KvBatch(s["starts"], s["kv_len"], s["table"], s["rows"], s["max_new"], s["max_len"])
        return s
    rows, vocab = case["rows"], case["vocab"]
    x = torch.randn(rows, vocab, device="cuda", generator=g) * 2.5
    likely = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    row = torch.arange(rows, device="cuda")
    x[row, likely] += 14 * torch.rand(rows, device="cuda", generator=g)
    other = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    tokens = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.6, likely, other)
    if case["hidden"]:  # tokens that a grammar rules out; the drafted one is allowed
        kept = x[row, tokens]
        x[torch.rand(rows, vocab, device="cuda", generator=g) < case["hidden"]] = -math.inf
        x[row, tokens] = kept
    s["logits"], s["tokens"] = x.to(t), tokens.to(torch.int32)
    return s


def run(s):
    if own:
        return _own(s)
    return {"groups": _groups, "rotate": _rotate, "tree": _tree, "scores": _scores}[s["kind"]](s)


def _own(s):
    from paper_2302_01382_amd import mpq

    if s["kind"] == "groups":
        act = {"none": mpq.ACT_NONE, "relu": mpq.ACT_RELU, "gelu": mpq.ACT_GELU}[s["act"]]
        return mpq.linear_groups(s["x"], s["w"], s["w_step"], act)
    if s["kind"] == "rotate":
        layout = mpq.ROTATE_PAIRS if s["pairs"] else mpq.ROTATE_HALVES
        return mpq.rotate_heads(s["q"], s["k"], s["positions"], s["frequencies"], s["q_weight"], s["k_weight"], EPS, layout)
    if s["kind"] == "tree":
        return mpq.kv_attention_tree(s["cache"], s["batch"], s["q"], s["tree"])
    return mpq.token_logprobs(s["logits"], s["tokens"], s["top"])


# ---- plain forms -------------------------------------------------------------------------------------------------------
def _groups(s):
    low, high = (s["w"] & 15).to(torch.int8), (s["w"] >> 4).to(torch.int8)
    codes = torch.stack([low, high], -1).flatten(1)
    codes = torch.where(codes > 7, codes - 16, codes).unflatten(1, (-1, s["group"]))
    w = (codes.float() * s["w_step"].float()[..., None]).flatten(1)
    y = s["x"].float() @ w.t()
    if s["act"] == "relu":
        y = torch.where(y > 0, y, torch.zeros_like(y))
    elif s["act"] == "gelu":
        y = (0.5 * y.double() * torch.erfc(y.double() * -math.sqrt(0.5))).float()
    return y.to(s["x"].dtype)


def _rotate(s):
    rot = s["rot"]
    # whole turns of far positions are dropped in 64 bits
    angle = s["positions"].double()[:, None] * s["frequencies"].double()
    angle = angle - torch.floor(angle / (2 * math.pi)) * (2 * math.pi)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = []
    for x, weight in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.float()
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / y.shape[-1] + EPS) * weight
        turned = y.clone()
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if s["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
        turned[..., a] = y[..., a] * cos - y[..., b] * sin
        turned[..., b] = y[..., b] * cos + y[..., a] * sin
        out.append(turned.to(x.dtype))
    return out


def _tree(s):
    heads, page, long, new = s["heads"], s["page"], s["max_len"], s["max_new"]
    group, dim, qmax = s["q_heads"] // heads, s["dim"], 2 ** (s["bits"] - 1) - 1
    starts, length = s["starts"].long(), s["kv_len"].long()
    i, out = torch.arange(new, device="cuda"), torch.zeros(s["rows"], s["q_heads"], dim, device="cuda")
    at_once = max(1, (1 << 29) // (long * heads * max(dim, group * new)))  # sequences, so that no tensor passes two gigabytes
    for first in range(0, s["seqs"], at_once):
        n = slice(first, first + at_once)
        j = torch.arange(long, device="cuda")
        pages = s["table"][n].long()[:, j // page]  # [sequences, places]
        k = s["k_codes"][pages, :, j % page].float() * (s["k_absmax"][pages] / qmax)[..., None]
        v = s["v_codes"][pages, :, j % page // 4, :, j % 4].float() * (s["v_absmax"][pages] / qmax)[..., None]
        begin, count = starts[:-1][n], (starts[1:] - starts[:-1])[n]
        rows = (begin[:, None] + i).clamp(max=s["rows"] - 1)  # past a sequence's end of no account
        q = s["q"][rows].float().unflatten(2, (heads, group)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [sequences, heads, group * new, dim]
        score = (q @ k.permute(0, 2, 3, 1).contiguous() * (1 / math.sqrt(dim))).unflatten(2, (group, new))
        drafted = j - (length[n] - count)[:, None]  # [sequences, places]: which drafted token, or before them
        word = (drafted.clamp(min=0) // 64).clamp(max=s["tree"].shape[1] - 1)
        bits = s["tree"][rows].gather(2, word[:, None].expand(-1, new, -1)) >> (drafted.clamp(min=0) % 64)[:, None] & 1
        seen = (drafted[:, None] < 0) | ((bits == 1) & (j < length[n][:, None])[:, None])
        score = score.masked_fill(~seen[:, None, None], -math.inf)
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        total = p.sum(-1, keepdim=True)
        o = p.flatten(2, 3) @ v.transpose(1, 2).contiguous()
        o = (o / torch.where(total > 0, total, torch.ones_like(total)).flatten(2, 3)).unflatten(2, (group, new))
        row = torch.arange(int(s["rows"]), device="cuda")
        seq = torch.searchsorted(starts[1:], row, right=True)
        mine = (seq >= first) & (seq < first + at_once)
        o = o[(seq - first).clamp(0, o.shape[0] - 1), :, :, (row - starts[seq]).clamp(max=new - 1)].flatten(1, 2)
        out = torch.where(mine[:, None, None], o, out)
    return out.to(s["q"].dtype)


def _scores(s):
    rows, vocab = s["logits"].shape
    column, out = torch.arange(vocab, device="cuda"), []
    at_once = max(1, (1 << 28) // vocab)
    for first in range(0, rows, at_once):
        x = s["logits"][first:first + at_once].float()
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        total = e.sum(1, keepdim=True)
        norm = torch.log(total)
        back = torch.where(e > 0, x - top, torch.zeros_like(x))
        entropy = norm[:, 0] - (e * back).sum(1) / total[:, 0]
        token = s["tokens"][first:first + at_once].long()[:, None]
        logprob = (x.gather(1, token) - top - norm)[:, 0]
        values, indices = [], []
        for _ in range(s["top"]):
            best = x.amax(1, keepdim=True)
            index = torch.where(x == best, column, vocab).amin(1, keepdim=True)  # ties: the lowest
            values.append(best - top - norm)
            indices.append(index)
            x = x.scatter(1, index, -math.inf)
        out.append((logprob, entropy, torch.cat(values, 1), torch.cat(indices, 1).to(torch.int32)))
    return [torch.cat(part) for part in zip(*out)]


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    el = SIZE[case["type"]]
    if case["kind"] == "groups":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": m * k * el + n * k // 2 + n * (k // case["group"]) * SIZE[case["steps"]] + m * n * el, "flops": 2 * m * n * k}
    if case["kind"] == "rotate":
        values = case["rows"] * (case["q_heads"] + case["heads"]) * case["dim"]
        # squares and their sum, the norm, the weight, a product and a sum of two for the rotation
        return {"bytes": 2 * values * el + 4 * case["rows"] + 8 * case["dim"] + 2 * case["rot"], "flops": 7 * values}
    if case["kind"] == "tree":
        new, held = _lengths(case)
        seen = _trees(case, new, 0)
        pairs = sum(a * b for a, b in zip(new, held)) + sum(bin(b).count("1") for b in seen)
        keys = sum(new) + sum(held)
        return {"bytes": 2 * sum(new) * case["q_heads"] * case["dim"] * el + 2 * keys * case["heads"] * (case["dim"] + 4 / case["page"]),
                "flops": 4 * pairs * case["q_heads"] * case["dim"]}
    values = case["rows"] * case["vocab"]
    # a maximum, a difference, an exponential, two sums
    return {"bytes": values * el + case["rows"] * (12 + 8 * case["top"]), "flops": 6 * values}


# ---- the definitions in 64 bits, by themselves -----------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "groups":
        w = s["w"].long()
        w = torch.stack([(w + 8) % 16 - 8, (w // 16 + 8) % 16 - 8], 2).reshape(case["n"], case["k"]).double()
        x, y = s["x"].double(), 0
        for i in range(case["k"] // case["group"]):
            part = slice(i * case["group"], (i + 1) * case["group"])
            y = y + torch.matmul(x[:, part], w[:, part].transpose(0, 1)) * s["w_step"][:, i].double()
        return y.clamp(min=0) if case["act"] == "relu" else y * torch.special.ndtr(y) if case["act"] == "gelu" else y
    if case["kind"] == "rotate":
        rot, out = case["rot"], []
        for x, weight in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
            x = x.double()
            y = x * torch.rsqrt(x.square().mean(2, keepdim=True) + EPS) * weight.double()
            head = y[..., :rot].unflatten(2, (rot // 2, 2) if case["pairs"] else (2, rot // 2))
            head = head if case["pairs"] else head.transpose(2, 3)
            turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), torch.outer(s["positions"].double(), s["frequencies"].double()))
            head = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn[:, None])
            head = head if case["pairs"] else head.transpose(2, 3)
            out.append(torch.cat([head.flatten(2), y[..., rot:]], 2))
        return out
    if case["kind"] == "tree":
        new, held = _lengths(case)
        page, heads, dim = case["page"], case["heads"], case["dim"]
        group, q, bits = case["q_heads"] // heads, 2.0 ** (case["bits"] - 1) - 1, _trees(case, new, seed)
        outs, at = [], 0
        for n, a, b in zip(range(case["seqs"]), new, held):
            table = s["table"][n, : -(-(a + b) // page)].long()
            k = (s["k_codes"][table].double() * (s["k_absmax"][table].double() / q)[..., None, None]).transpose(0, 1).reshape(heads, -1, dim)[:, : a + b]
            v = s["v_codes"][table].double() * (s["v_absmax"][table].double() / q)[..., None, None, None]
            v = v.permute(1, 0, 2, 4, 3).reshape(heads, -1, dim)[:, : a + b]
            hidden = torch.zeros(a, a + b, dtype=torch.bool)
            hidden[:, b:] = torch.tensor([[not bits[at + i] >> j & 1 for j in range(a)] for i in range(a)])
            hidden = hidden.to("cuda")
            o = torch.empty(a, case["q_heads"], dim, dtype=torch.float64, device="cuda")
            for h in range(case["q_heads"]):
                logits = torch.mm(s["q"][at:at + a, h].double(), k[h // group].t()) / math.sqrt(dim)
                o[:, h] = torch.softmax(logits.masked_fill_(hidden, -math.inf), 1).mm(v[h // group])
            outs.append(o)
            at += a
        return torch.cat(outs)
    out = []
    for first in range(0, case["rows"], 256):
        x = s["logits"][first:first + 256].double()
        p = torch.log_softmax(x, 1)
        entropy = torch.special.entr(p.exp()).sum(1)
        order = torch.sort(x, dim=1, descending=True, stable=True)
        top = order.indices[:, : case["top"]]
        out.append((p.gather(1, s["tokens"][first:first + 256].long()[:, None])[:, 0], entropy, p.gather(1, top), top.int()))
    return [torch.cat(part) for part in zip(*out)]
