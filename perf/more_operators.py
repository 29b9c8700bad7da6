"""Cases, inputs and plain forms of four operators with which a model in training writes the answers that it then learns from:

  rotary   rotary positions: a table of angles, scaled for long contexts or not, and the rotation of heads by it, forward and backward
  append   a batch's new tokens on their way into a paged cache: queries and keys rotated, keys and values written to their pages
  attend   attention of the new tokens over the cache, from one token a sequence to chunks of a prompt
  adjust   penalties for tokens that a row has seen, a bias and a grammar's mask on logits, and the gradient through them

With `own` true `run` calls the framework's kernels, otherwise elementary torch operations in 32 bits (the table's angles in 64)."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
ROTARY = dict(plain=dict(scaling="plain"), linear=dict(scaling="linear", factor=4.0), base=dict(scaling="base", factor=8.0),
              parts=dict(scaling="parts", factor=16.0, trained=4096.0, slow=1.0, fast=32.0, amplitude=1.2772588722239782))


def listed():
    return [
        # queries and keys of one token in flight for each of four sequences, neighbouring columns paired, half of each head: latency
        dict(name="rotary four tokens", op="rotary", what="rows", rows=4, heads=40, head_dim=128, rot=64, layout="pairs", backward=False, given=True, dtype="bf16"),
        # gradients of q and k of a 7B layer, 4 x 512 tokens, inside the gradient of the fused projection
        dict(name="rotary 7B batch backward", op="rotary", what="rows", rows=2048, heads=64, head_dim=128, rot=128, layout="halves", backward=True, given=False, dtype="bf16"),
        # the angles of a context sixteen times as long as trained on
        dict(name="rotary long table", op="rotary", what="table", count=65536, rot=128, base=10000.0, scaling="parts"),
        # 64 answers in the making, a token each, grouped heads: latency
        dict(name="append one token each", op="append", seqs=64, new=1, new_min=1, cached=4000, cached_min=1, heads=32, kv_heads=8, head_dim=128, rot=128,
             layout="halves", page=16, dtype="bf16"),
        # prompts of different lengths at the 7B widths, into empty and half-filled caches
        dict(name="append prompts", op="append", seqs=8, new=1000, new_min=33, cached=500, cached_min=0, heads=32, kv_heads=32, head_dim=128, rot=128,
             layout="halves", page=64, dtype="bf16"),
        # the next token of one answer at the 7B widths: latency
        dict(name="attend one token", op="attend", seqs=1, new=1, new_min=1, cached=500, cached_min=500, heads=32, kv_heads=32, head_dim=128, page=16, window=0,
             dtype="bf16"),
        # 64 answers of all lengths, grouped heads
        dict(name="attend answers", op="attend", seqs=64, new=1, new_min=1, cached=8000, cached_min=1, heads=32, kv_heads=8, head_dim=128, page=16, window=0,
             dtype="bf16"),
        # chunks of long prompts at the 7B widths
        dict(name="attend chunks", op="attend", seqs=4, new=1024, new_min=700, cached=4096, cached_min=0, heads=32, kv_heads=32, head_dim=128, page=64, window=0,
             dtype="bf16"),
        # a small fp32 model, a few tokens each, heads of an odd width, a sliding window
        dict(name="attend fp32 window", op="attend", seqs=3, new=77, new_min=1, cached=901, cached_min=5, heads=8, kv_heads=2, head_dim=80, page=32, window=256,
             dtype="fp32"),
        # the next token of one answer, penalties alone: latency
        dict(name="adjust one row", op="adjust", rows=1, vocab=32000, history=300, nested=False, bias=False, mask="none", backward=False, dtype="bf16"),
        # answers under a grammar of their own each, a vocabulary that leaves rows unaligned
        dict(name="adjust odd vocabulary", op="adjust", rows=256, vocab=50265, history=1500, nested=False, bias=True, mask="rows", backward=False, dtype="bf16"),
        # a scored 7B batch, 4 x 512 tokens: every position has seen what precedes it, banned tokens for all
        dict(name="adjust gradient 7B batch", op="adjust", rows=2048, vocab=32000, history=511, nested=True, bias=True, mask="one", backward=True, dtype="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {"rotary": 1e8, "append": 2.2e8, "attend": 1.1e9, "adjust": 2.7e8}
    while True:
        op, dtype = rng.choice(["rotary", "append", "attend", "attend", "adjust"]), rng.choice(["bf16", "fp32"])
        if op == "rotary" and rng.random() < 0.3:
            case = dict(op=op, what="table", count=log_int(1, 65536), rot=2 * rng.randint(1, 64), base=rng.choice([10000.0, 500000.0]),
                        scaling=rng.choice(["plain", "linear", "base", "parts"]))
            case["rot"] = max(case["rot"], 4)
        elif op == "rotary":
            head_dim = rng.choice([16, 32, 64, 80, 96, 128, 256, 2 * rng.randint(1, 100)])
            rot = rng.choice([head_dim, head_dim, max(2, head_dim // 4 * 2)])
            case = dict(op=op, what="rows", rows=log_int(1, 8192), heads=log_int(1, 80), head_dim=head_dim, rot=rot, layout=rng.choice(["halves", "pairs"]),
                        backward=rng.random() < 0.5, given=rng.random() < 0.5, dtype=dtype)
        elif op == "adjust":
            case = dict(op=op, rows=log_int(1, 4096), vocab=log_int(100, 130000), history=log_int(1, 8192), nested=rng.random() < 0.3, bias=rng.random() < 0.5,
                        mask=rng.choice(["none", "rows", "one"]), backward=rng.random() < 0.4, dtype=dtype)
            if case["nested"]:
                case["history"] = min(case["history"], 1023)
            if case["rows"] * case["history"] > 2 ** 21:
                continue
        else:
            kv_heads, head_dim = rng.choice([1, 2, 4, 8, 16, 32]), rng.choice([16, 32, 64, 80, 96, 128, 128])
            case = dict(op=op, seqs=log_int(1, 128), new=1 if rng.random() < 0.4 else log_int(2, 1024), new_min=1, cached=log_int(1, 16384), cached_min=rng.choice([0, 1]),
                        heads=min(64, kv_heads * rng.choice([1, 2, 4, 8])), kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([16, 32, 64, 128]), dtype=dtype)
            if op == "append":
                case.update(rot=rng.choice([head_dim, max(2, head_dim // 4 * 2)]), layout=rng.choice(["halves", "pairs"]), cached=min(case["cached"], 4096))
            else:
                case.update(window=rng.choice([0, 0, 0, log_int(1, 4096)]))
            # what the plain form widens to 32 bits fits the card
            pool = case["seqs"] * (case["cached"] + case["new"]) * kv_heads * head_dim
            if pool > 5e8 or (op == "attend" and case["seqs"] * case["new"] * case["heads"] * (case["cached"] + case["new"]) > 8e8):
                continue
        w = work(case)
        if w["bytes"] <= most[op] and w["flops"] <= (2e11 if dtype == "bf16" or op != "attend" else 1.5e10):
            return case


def spread(lo, hi, n, turn):
    """n whole numbers from lo to hi, in an order that does not rise."""
    if n == 1:
        return [hi]
    return [lo + round((hi - lo) * ((i * turn) % n) / (n - 1)) for i in range(n)]


def tokens_of(case):
    """(cached, new) of every sequence."""
    n = case["seqs"]
    turn = next(t for t in (max(1, n * 5 // 13), 7, 11, 3, 1) if math.gcd(t, n) == 1)
    return list(zip(spread(case["cached_min"], case["cached"], n, turn), spread(case["new_min"], case["new"], n, 1)))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return dict(case, **{"rotary": prepare_rotary, "append": prepare_cache, "attend": prepare_cache, "adjust": prepare_adjust}[case["op"]](case, g))


def some_table(rows, rot):
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    return torch.stack([angle.cos(), angle.sin()], 2).float()


def prepare_rotary(case, g):
    if case["what"] == "table":
        first = int(torch.randint(0, 1000, (1,), generator=g, device="cuda"))
        return dict(first=first, rotary=dict(ROTARY[case["scaling"]], rot=case["rot"], base=case["base"]),
                    cos_sin=torch.empty(case["count"], case["rot"] // 2, 2, device="cuda"))
    rows, width, dt = case["rows"], case["heads"] * case["head_dim"], DTYPES[case["dtype"]]
    # rows of a fused projection: what follows the rotated heads stays where it is
    x = torch.randn(rows, width + width // 2, generator=g, device="cuda").to(dt)
    seq = 512
    s = dict(x=x[:, :width], y=torch.empty(rows, width, device="cuda", dtype=dt), seq=seq, cos_sin=some_table(4096 if case["given"] else seq, case["rot"]), positions=None)
    if case["given"]:
        s["positions"] = torch.randint(0, 4096, (rows,), generator=g, device="cuda", dtype=torch.int32)
    return s


def prepare_cache(case, g):
    tokens, page, dt = tokens_of(case), case["page"], DTYPES[case["dtype"]]
    kv, hd = case["kv_heads"], case["head_dim"]
    need = [-(-(c + n) // page) for c, n in tokens]
    most, pool = max(need), sum(need) + 3
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    pages = torch.full((case["seqs"], most), -1, device="cuda", dtype=torch.int32)
    used = 0
    for i, n in enumerate(need):
        pages[i, :n] = order[used:used + n]
        used += n
    starts = [0]
    for _, n in tokens:
        starts.append(starts[-1] + n)
    rows = starts[-1]
    s = dict(pages=pages, starts=torch.tensor(starts, device="cuda", dtype=torch.int32), lengths=torch.tensor([c for c, _ in tokens], device="cuda", dtype=torch.int32),
             max_new=max(n for _, n in tokens), max_length=max(c + n for c, n in tokens),
             k=torch.randn(pool, kv, page, hd, generator=g, device="cuda", dtype=dt), v=torch.randn(pool, kv, page, hd, generator=g, device="cuda", dtype=dt))
    if case["op"] == "append":
        s["qkv"] = torch.randn(rows, (case["heads"] + 2 * kv) * hd, generator=g, device="cuda", dtype=dt)
        s["q"] = torch.empty(rows, case["heads"] * hd, device="cuda", dtype=dt)
        s["cos_sin"] = some_table(max(c + n for c, n in tokens), case["rot"])
    else:
        # queries that prefer some keys, as trained heads do
        s["q"] = torch.randn(rows, case["heads"] * hd, generator=g, device="cuda", dtype=dt) * 1.5
        s["out"], s["lse"] = torch.empty(rows, case["heads"] * hd, device="cuda", dtype=dt), torch.empty(rows, case["heads"], device="cuda")
    if own:
        import paper_2401_15207_amd as H
        s["cache"] = H.PagedCache(s["k"], s["v"], s["pages"], s["lengths"])
        if case["op"] == "attend":
            n = H.kernel_attention_paged_bytes(s["cache"], rows, case["heads"], s["max_new"], s["max_length"], window=case["window"])
            s["workspace"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    return s


def prepare_adjust(case, g):
    rows, vocab, dt, most = case["rows"], case["vocab"], DTYPES[case["dtype"]], case["history"]
    if case["nested"]:
        # positions of texts: each has seen its text up to itself
        texts = -(-rows // (most + 1))
        count = texts * (most + 1)
        at = torch.arange(rows, device="cuda")
        begin = at // (most + 1) * (most + 1)
        end = at + 1
        seen = [i % (most + 1) + 1 for i in range(rows)]
    else:
        seen = spread(0, most, rows, next(t for t in (7, 5, 11, 1) if math.gcd(t, rows) == 1))
        end = torch.tensor(seen, device="cuda").cumsum(0)
        begin = end - torch.tensor(seen, device="cuda")
        count = sum(seen)
    # texts repeat themselves: few tokens often, most of them hardly ever
    tokens = (torch.rand(count, generator=g, device="cuda") ** 4 * vocab).long().clamp(max=vocab - 1)
    tokens = tokens * 7919 % vocab
    s = dict(tokens=tokens.to(torch.int32), begin=begin, end=end, total=sum(seen), repetition=1.2, presence=0.4, frequency=0.1, bias_row=None, allowed=None)
    logits = torch.randn(rows, vocab, generator=g, device="cuda").mul_(2.5)
    s["logits"] = logits.to(dt)
    if case["bias"]:
        s["bias_row"] = torch.randn(1, vocab, generator=g, device="cuda") * (torch.rand(1, vocab, generator=g, device="cuda") < 0.05)
    if case["mask"] != "none":
        words = (1 if case["mask"] == "one" else rows, -(-vocab // 32))
        a, b = (torch.randint(-2 ** 31, 2 ** 31, words, generator=g, device="cuda", dtype=torch.int64).to(torch.int32) for _ in range(2))
        # a grammar lets few tokens through, a list of banned ones most
        s["allowed"] = a & b if case["mask"] == "rows" else a | b
    if case["backward"]:
        s["d_out"] = (torch.randn(rows, vocab, generator=g, device="cuda") / rows).to(dt)
        s["d_logits"] = torch.empty_like(s["logits"])
    else:
        s["out"] = torch.empty_like(s["logits"])
    return s


def run(s):
    return (own_form if own else plain_form)[s["op"]](s)


# ---- the framework's operators ----
def own_rotary(s):
    import paper_2401_15207_amd as H
    if s["what"] == "table":
        H.kernel_rotary_table(s["rotary"], s["cos_sin"], first=s["first"])
        return s["cos_sin"]
    H.kernel_rotary(s["x"], s["heads"], s["head_dim"], s["y"], s["cos_sin"], positions=s["positions"], seq=s["seq"], layout=s["layout"], backward=s["backward"])
    return s["y"]


def own_append(s):
    import paper_2401_15207_amd as H
    H.kernel_cache_append(s["cache"], s["starts"], s["qkv"], s["heads"], s["q"], s["cos_sin"], layout=s["layout"], max_new=s["max_new"])
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def own_attend(s):
    import paper_2401_15207_amd as H
    H.kernel_attention_paged(s["cache"], s["starts"], s["q"], s["heads"], s["out"], max_new=s["max_new"], max_length=s["max_length"], window=s["window"], lse=s["lse"],
                             workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def own_adjust(s):
    import paper_2401_15207_amd as H
    more = dict(repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"], bias=s["bias_row"], allowed=s["allowed"])
    if s["backward"]:
        H.kernel_adjust_logits_bwd(s["logits"], s["vocab"], s["d_out"], s["d_logits"], s["tokens"], s["begin"], s["end"], **more)
        return s["d_logits"]
    H.kernel_adjust_logits(s["logits"], s["vocab"], s["out"], s["tokens"], s["begin"], s["end"], **more)
    return s["out"]


# ---- their plain forms ----
def plain_rates(r):
    """Angle by position of each pair, in 64 bits."""
    i = torch.arange(0, r["rot"], 2, device="cuda", dtype=torch.float64)
    base = r["base"] * r["factor"] ** (r["rot"] / (r["rot"] - 2)) if r["scaling"] == "base" else r["base"]
    rate = base ** (-i / r["rot"])
    if r["scaling"] == "linear":
        rate = rate / r["factor"]
    if r["scaling"] == "parts":
        turns = r["trained"] * rate / (2.0 * math.pi)
        keep = ((turns - r["slow"]) / (r["fast"] - r["slow"])).clamp(0.0, 1.0)
        rate = rate * keep + rate / r["factor"] * (1.0 - keep)
    return rate


def plain_rotate(x, cs, layout, backward):
    """x [rows, heads, head_dim] in 32 bits, cs [rows, rot / 2, 2]."""
    half = cs.shape[1]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    sin = -sin if backward else sin
    if layout == "halves":
        a, b = x[..., :half], x[..., half:2 * half]
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    a, b = a * cos - b * sin, b * cos + a * sin
    y = x.clone()
    if layout == "halves":
        y[..., :half], y[..., half:2 * half] = a, b
    else:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a, b
    return y


def plain_rotary(s):
    if s["what"] == "table":
        r = s["rotary"]
        at = torch.arange(s["first"], s["first"] + s["count"], device="cuda", dtype=torch.float64)
        angle = at[:, None] * plain_rates(r)
        return (torch.stack([angle.cos(), angle.sin()], 2) * r.get("amplitude", 1.0)).float()
    rows = s["rows"]
    at = torch.arange(rows, device="cuda") % s["seq"] if s["positions"] is None else s["positions"].long()
    y = plain_rotate(s["x"].float().view(rows, s["heads"], s["head_dim"]), s["cos_sin"][at], s["layout"], s["backward"])
    return y.to(s["x"].dtype).view(rows, -1)


def plain_places(s, rows):
    """Sequence and place within its new rows of every row."""
    at = torch.arange(rows, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["starts"], at, right=True) - 1
    return seq, at.long() - s["starts"][seq].long()


def plain_append(s):
    rows, heads, kv, hd, page = s["qkv"].shape[0], s["heads"], s["kv_heads"], s["head_dim"], s["page"]
    seq, place = plain_places(s, rows)
    at = s["lengths"][seq].long() + place
    cs = s["cos_sin"][at]
    x = s["qkv"].view(rows, heads + 2 * kv, hd)
    turned = plain_rotate(x[:, :heads + kv].float(), cs, s["layout"], False).to(x.dtype)
    to = s["pages"][seq, at // page].long()
    s["k"][to, :, at % page] = turned[:, heads:]
    s["v"][to, :, at % page] = x[:, heads + kv:]
    return {"q": turned[:, :heads].reshape(rows, -1), "k": s["k"], "v": s["v"]}


def plain_attend(s):
    rows, heads, kv, hd, new = s["q"].shape[0], s["heads"], s["kv_heads"], s["head_dim"], s["max_new"]
    n, group = s["seqs"], s["heads"] // s["kv_heads"]
    to = s["pages"].long().clamp(min=0)
    k, v = (t[to].float().transpose(1, 2).reshape(n, kv, -1, hd) for t in (s["k"], s["v"]))
    first, count = s["starts"][:-1].long(), (s["starts"][1:] - s["starts"][:-1]).long()
    place = torch.arange(new, device="cuda")
    q = s["q"].float().view(rows, kv, group, hd)[(first[:, None] + place).clamp(max=rows - 1)]
    q = q.permute(0, 2, 3, 1, 4).reshape(n, kv, group * new, hd)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).view(n, kv, group, new, -1) * (1.0 / math.sqrt(hd))
    at = (s["lengths"].long()[:, None] + place)[:, None, None, :, None]
    key = torch.arange(k.shape[2], device="cuda")
    seen = (key <= at) & (key < (s["lengths"].long() + count)[:, None, None, None, None])
    if s["window"]:
        seen = seen & (key > at - s["window"])
    score = torch.where(seen, score, -math.inf)
    top = score.max(-1, keepdim=True).values
    e = torch.exp(score - top)
    total = e.sum(-1, keepdim=True)
    out = torch.matmul((e / total).view(n, kv, group * new, -1), v).view(n, kv, group, new, hd)
    lse = (top + total.log()).squeeze(-1) * (1.0 / math.log(2.0))
    seq, place = plain_places(s, rows)
    return {"out": out[seq, :, :, place].reshape(rows, -1).to(s["q"].dtype), "lse": lse[seq, :, :, place].reshape(rows, heads)}


def plain_counts(s):
    """How often each row has seen each token."""
    rows = s["rows"]
    row = torch.repeat_interleave(torch.arange(rows, device="cuda"), s["end"] - s["begin"], output_size=s["total"])
    before = (s["end"] - s["begin"]).cumsum(0) - (s["end"] - s["begin"])
    token = s["tokens"][torch.arange(s["total"], device="cuda") - before[row] + s["begin"][row]].long()
    counts = torch.zeros(rows, s["vocab"], device="cuda")
    return counts.index_put_((row, token), torch.ones((), device="cuda"), accumulate=True)


def plain_allowed(s):
    bits = (s["allowed"].unsqueeze(-1) >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    return bits.flatten(1)[:, :s["vocab"]].bool()


def plain_adjust(s):
    x, counts = s["logits"].float(), plain_counts(s)
    if s["backward"]:
        d = s["d_out"].float()
        d = torch.where(counts > 0, torch.where(x > 0, d / s["repetition"], d * s["repetition"]), d)
        return (d if s["allowed"] is None else torch.where(plain_allowed(s), d, 0.0)).to(s["logits"].dtype)
    z = torch.where(counts > 0, torch.where(x > 0, x / s["repetition"], x * s["repetition"]) - s["presence"], x) - s["frequency"] * counts
    if s["bias_row"] is not None:
        z = z + s["bias_row"]
    return (z if s["allowed"] is None else torch.where(plain_allowed(s), z, -math.inf)).to(s["logits"].dtype)


own_form = {"rotary": own_rotary, "append": own_append, "attend": own_attend, "adjust": own_adjust}
plain_form = {"rotary": plain_rotary, "append": plain_append, "attend": plain_attend, "adjust": plain_adjust}


def work(case):
    if case["op"] == "rotary" and case["what"] == "table":
        return {"bytes": case["count"] * case["rot"] * 4.0, "flops": 40.0 * case["count"] * case["rot"]}
    size = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "rotary":
        table = (min(case["rows"], 4096) if case["given"] else min(case["rows"], 512)) * case["rot"] * 4
        return {"bytes": 2.0 * case["rows"] * case["heads"] * case["head_dim"] * size + table + (4 * case["rows"] if case["given"] else 0),
                "flops": 3.0 * case["rows"] * case["heads"] * case["rot"]}
    if case["op"] == "adjust":
        rows, vocab = case["rows"], case["vocab"]
        seen = case["history"] + 1 if case["nested"] else case["history"] / 2
        masks = {"none": 0, "one": 1, "rows": rows}[case["mask"]] * vocab / 8
        history = 4.0 * rows if case["nested"] else 4.0 * rows * seen
        # forward every line of the logits is read, since allowed tokens lie scattered; the gradient needs the logits of seen tokens alone
        return {"bytes": rows * vocab * size * 2.0 + (rows * min(seen, vocab) * size if case["backward"] else 0) + masks + history + (4.0 * vocab if case["bias"] and not case["backward"] else 0), "flops": 6.0 * rows * vocab}
    tokens, heads, kv, hd = tokens_of(case), case["heads"], case["kv_heads"], case["head_dim"]
    rows = sum(n for _, n in tokens)
    if case["op"] == "append":
        table = len({c + i for c, n in tokens for i in range(n)}) * case["rot"] * 4
        return {"bytes": 2.0 * rows * (heads + 2 * kv) * hd * size + table, "flops": 3.0 * rows * (heads + kv) * case["rot"]}
    keys = pairs = 0
    for c, n in tokens:
        w = case["window"] or c + n
        keys += min(c + n, n - 1 + w)
        pairs += sum(min(c + i + 1, w) for i in range(n))
    return {"bytes": 2.0 * keys * kv * hd * size + 2.0 * rows * heads * hd * size + 4.0 * rows * heads, "flops": 4.0 * pairs * heads * hd}


# ---- from the definitions, in 64 bits ----
def exact_turned(x, cs, layout, backward):
    """A pair is a complex number, its rotation a product with cos + i sin (backward: with its conjugate)."""
    half = cs.shape[-2]
    turn = torch.view_as_complex(cs.double().contiguous())
    turn = (turn.conj() if backward else turn).unsqueeze(-2)
    y = x.double().clone()
    at = torch.arange(half, device=x.device)
    one, two = (at, at + half) if layout == "halves" else (2 * at, 2 * at + 1)
    z = torch.complex(y[..., one], y[..., two]) * turn
    y[..., one], y[..., two] = z.real, z.imag
    return y


def exact_rotary(case, s):
    if case["what"] == "table":
        r, rates = s["rotary"], []
        for i in range(case["rot"] // 2):
            base = r["base"] * (r["factor"] ** (r["rot"] / (r["rot"] - 2.0)) if r["scaling"] == "base" else 1.0)
            rate = math.exp(-2.0 * i / r["rot"] * math.log(base))
            if r["scaling"] == "linear":
                rate /= r["factor"]
            elif r["scaling"] == "parts":
                keep = min(1.0, max(0.0, (rate * r["trained"] / (2 * math.pi) - r["slow"]) / (r["fast"] - r["slow"])))
                rate = (1 - keep) * rate / r["factor"] + keep * rate
            rates.append(rate)
        angle = torch.outer(torch.arange(case["count"], dtype=torch.float64) + s["first"], torch.tensor(rates, dtype=torch.float64))
        return (torch.view_as_real(torch.polar(torch.full_like(angle, r.get("amplitude", 1.0)), angle))).cuda()
    rows = case["rows"]
    at = s["positions"].long() if case["given"] else torch.arange(rows, device="cuda") % s["seq"]
    return exact_turned(s["x"].reshape(rows, case["heads"], case["head_dim"]), s["cos_sin"][at], case["layout"], case["backward"]).view(rows, -1)


def exact_append(case, s):
    heads, kv, hd, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    k, v, q, row = s["k"].double(), s["v"].double(), [], 0
    pages = s["pages"].long()
    for i, (cached, new) in enumerate(tokens_of(case)):
        x = s["qkv"][row:row + new].double().view(new, heads + 2 * kv, hd)
        at = torch.arange(cached, cached + new, device="cuda")
        turned = exact_turned(x[:, :heads + kv], s["cos_sin"][cached:cached + new], case["layout"], False)
        k[pages[i, at // page], :, at % page] = turned[:, heads:]
        v[pages[i, at // page], :, at % page] = x[:, heads + kv:]
        q.append(turned[:, :heads].reshape(new, -1))
        row += new
    return {"q": torch.cat(q), "k": k, "v": v}


def exact_attend(case, s):
    heads, kv, hd, page = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    out, lse, row = [], [], 0
    for i, (cached, new) in enumerate(tokens_of(case)):
        have = cached + new
        used = s["pages"][i, :-(-have // page)].long()
        k, v = (t[used].double().permute(1, 0, 2, 3).reshape(kv, -1, hd)[:, :have].contiguous() for t in (s["k"], s["v"]))
        q = s["q"][row:row + new].double().view(new, heads, hd).transpose(0, 1).contiguous()
        low = torch.zeros(have, new, device="cuda", dtype=torch.float64)
        key, at = torch.arange(have, device="cuda")[:, None], torch.arange(cached, have, device="cuda")[None, :]
        low.masked_fill_((key > at) | ((key <= at - case["window"]) if case["window"] else False), -math.inf)
        o, z = [], []
        for h in range(heads):
            kh, vh = k[h // (heads // kv)], v[h // (heads // kv)]
            score = torch.mm(kh, q[h].t().contiguous()) / math.sqrt(hd) + low
            z.append(torch.logsumexp(score, 0))
            o.append(torch.mm(torch.exp(score - z[-1]).t().contiguous(), vh))
        out.append(torch.stack(o, 1).reshape(new, heads * hd))
        lse.append(torch.stack(z, 1) / math.log(2.0))
        row += new
    return {"out": torch.cat(out), "lse": torch.cat(lse)}


def exact_adjust(case, s):
    rows, vocab = case["rows"], case["vocab"]
    x = s["logits"].double()
    counts = torch.stack([torch.bincount(s["tokens"][b:e].long(), minlength=vocab) for b, e in zip(s["begin"].tolist(), s["end"].tolist())]).to(torch.float64)
    factor = torch.where(counts > 0, torch.where(x > 0, 1.0 / s["repetition"], s["repetition"]), 1.0)
    banned = None
    if s["allowed"] is not None:
        at = torch.arange(vocab, device="cuda")
        banned = (s["allowed"].long() & 0xFFFFFFFF)[:, at // 32] // 2 ** (at % 32) % 2 == 0
        banned = banned.expand(rows, vocab)
    if case["backward"]:
        d = s["d_out"].double() * factor
        return d if banned is None else d.masked_fill(banned, 0.0)
    z = x * factor - s["presence"] * counts.clamp(max=1.0) - s["frequency"] * counts
    z = z if s["bias_row"] is None else z + s["bias_row"].double()
    return z if banned is None else z.masked_fill(banned, -math.inf)


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": exact_rotary, "append": exact_append, "attend": exact_attend, "adjust": exact_adjust}[case["op"]](case, s)
