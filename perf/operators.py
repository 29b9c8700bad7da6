"""Cases, inputs and plain forms of four operators of a fine-tuning step that learns from scored tokens:

  logprob      log probabilities of given tokens with the entropy of each row and its most probable alternatives
  logprob_bwd  gradient of the log probabilities and of the entropy with respect to the logits
  ortho        orthogonalisation of update matrices by five Newton-Schulz steps
  muon         update of a group's matrices: momentum, orthogonalised step, decay, master weights and their bf16 copy

With `own` true `run` calls the framework's kernels, otherwise elementary torch operations in 32 bits."""
import math

import torch

own = False

STEPS, COEF, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def shapes_of(case):
    return [tuple(int(x) for x in s.split("x")) for s in case["shapes"].split(",")]


def listed():
    layer_1024 = "1024x1024,1024x1024,1024x1024,1024x1024,4096x1024,1024x4096"
    layer_4096 = "4096x4096,4096x4096,4096x4096,4096x4096,11008x4096,11008x4096,4096x11008"
    return [
        # one sequence's next token while an answer is sampled: latency
        dict(name="logprob one row", op="logprob", rows=1, vocab=32000, pad=0, dtype="bf16", top=20, temperature=0.8, masked=0.0, empty=0.0),
        # a scored batch whose vocabulary leaves rows unaligned, some tokens banned, some positions without a target
        dict(name="logprob odd vocabulary", op="logprob", rows=777, vocab=50265, pad=0, dtype="bf16", top=5, temperature=0.7, masked=0.02, empty=0.1),
        # a training batch of the 7B shape, 4 x 512 tokens
        dict(name="logprob 7B batch", op="logprob", rows=2048, vocab=32000, pad=0, dtype="bf16", top=8, temperature=1.0, masked=0.0, empty=0.01),
        # evaluation of a long batch with fp32 logits, no alternatives asked for
        dict(name="logprob fp32 batch", op="logprob", rows=4096, vocab=50272, pad=0, dtype="fp32", top=0, temperature=1.0, masked=0.0, empty=0.01),
        # the tiny decoder: 2 x 32 tokens, 256 entries
        dict(name="gradient tiny", op="logprob_bwd", rows=64, vocab=256, pad=0, dtype="fp32", top=0, temperature=1.0, masked=0.0, empty=0.1),
        # half of a scored batch, unaligned rows, banned tokens
        dict(name="gradient odd vocabulary", op="logprob_bwd", rows=1000, vocab=50265, pad=0, dtype="bf16", top=0, temperature=0.7, masked=0.02, empty=0.1),
        dict(name="gradient 7B batch", op="logprob_bwd", rows=2048, vocab=32000, pad=0, dtype="bf16", top=0, temperature=1.0, masked=0.0, empty=0.01),
        # the six matrices of a layer of the tiny decoder: latency
        dict(name="ortho tiny layer", op="ortho", shapes="64x64,64x64,64x64,64x64,256x64,64x256", dtype="fp32", out="fp32"),
        # matrices whose sides are no multiple of anything
        dict(name="ortho odd sizes", op="ortho", shapes="1000x333,129x257,77x1300,515x515", dtype="bf16", out="fp32"),
        # a layer 1024 wide with 4096 in its feed-forward block
        dict(name="ortho 1024 layer", op="ortho", shapes=layer_1024, dtype="fp32", out="bf16"),
        dict(name="muon 1024 layer", op="muon", shapes=layer_1024, lr=5e-5, momentum=0.95, decay=0.01),
        # a hidden layer of the 7B shape: the group of one step
        dict(name="muon 7B layer", op="muon", shapes=layer_4096, lr=1e-5, momentum=0.95, decay=0.0),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["logprob", "logprob_bwd", "ortho", "muon"])
    if op.startswith("logprob"):
        dtype = rng.choice(["bf16", "fp32"])
        vocab = log_int(100, 130000)
        rows = min(log_int(1, 8192), max(1, (100 if dtype == "fp32" else 200) * 10 ** 6 // vocab))
        return dict(op=op, rows=rows, vocab=vocab, pad=rng.choice([0, 0, 0, 1, 7, 8]), dtype=dtype,
                    top=rng.choice([0, 1, 5, 8, 20, 32]) if op == "logprob" else 0, temperature=rng.choice([0.5, 0.7, 1.0, 1.3]),
                    masked=rng.choice([0.0, 0.02, 0.5]), empty=rng.choice([0.0, 0.01, 0.2]))
    limit, shapes, cost = 2e12, [], 0.0
    for _ in range(rng.randint(1, 7)):
        r, c = log_int(8, 8192), log_int(8, 8192)
        n, m = min(r, c), max(r, c)
        cost += STEPS * (3.0 * n * n * m + n ** 3)
        if cost > limit and shapes:
            break
        shapes.append("%dx%d" % ((r, c) if cost <= limit else (r // 2 + 4, c // 2 + 4)))
    if op == "ortho":
        return dict(op=op, shapes=",".join(shapes), dtype=rng.choice(["bf16", "fp32"]), out=rng.choice(["bf16", "fp32"]))
    return dict(op=op, shapes=",".join(shapes), lr=rng.choice([1e-5, 2e-5, 8e-5]), momentum=rng.choice([0.9, 0.95]), decay=rng.choice([0.0, 0.01]))


def gradient_like(g, r, c):
    """A few strong directions over a floor of noise, at the scale of a fine-tuning gradient."""
    k = min(16, r, c)
    u = torch.randn(r, k, generator=g, device="cuda") * torch.logspace(0.0, -1.5, k, device="cuda")
    return (u @ torch.randn(k, c, generator=g, device="cuda") + 0.3 * torch.randn(r, c, generator=g, device="cuda")) * 1e-4


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["op"].startswith("logprob"):
        rows, vocab, dt = case["rows"], case["vocab"], DTYPES[case["dtype"]]
        ld = vocab + case["pad"]
        # logits of a trained model: a wide body and a few tokens far above it
        logits = torch.randn(rows, ld, generator=g, device="cuda").mul_(1.7)
        peaks = (torch.randint(0, vocab, (rows, 1), generator=g, device="cuda") + torch.arange(12, device="cuda") * (vocab // 12)) % vocab
        logits.scatter_add_(1, peaks, torch.rand(rows, 12, generator=g, device="cuda") * 9.0)
        if case["masked"]:
            logits.masked_fill_(torch.rand(ld, generator=g, device="cuda") < case["masked"], -math.inf)
        s["logits"] = logits.to(dt)
        targets = peaks[:, 0].clone()
        targets[torch.rand(rows, generator=g, device="cuda") < case["empty"]] = -1
        # a banned token is never the one that was chosen
        chosen = logits.gather(1, targets.clamp(min=0).unsqueeze(1)).squeeze(1)
        s["targets"] = torch.where(torch.isinf(chosen), -1, targets).to(torch.int32)
        s["scale"] = 1.0 / case["temperature"]
        if case["op"] == "logprob_bwd":
            s["d_logp"] = torch.randn(rows, generator=g, device="cuda") / rows
            s["d_entropy"] = 0.01 * torch.rand(rows, generator=g, device="cuda") / rows
            z = s["logits"][:, :vocab].float() * s["scale"]  # what the forward pass left
            top = z.max(1, keepdim=True).values
            top = torch.where(torch.isinf(top), 0.0, top)
            e = torch.exp(z - top)
            total = e.sum(1)
            s["stats"] = torch.stack([top.squeeze(1), total.log()], 1).contiguous()
            s["entropy"] = total.log() - torch.where(e > 0, e * (z - top), 0.0).sum(1) / total
            del z, e
            s["dlogits"] = torch.empty_like(s["logits"])
        else:
            f = dict(device="cuda", dtype=torch.float32)
            s["logp"], s["entropy"], s["stats"] = torch.empty(rows, **f), torch.empty(rows, **f), torch.empty(rows, 2, **f)
            s["top_logp"] = torch.empty(rows, case["top"], **f)
            s["top_ids"] = torch.empty(rows, case["top"], device="cuda", dtype=torch.int32)
        return s
    shapes = shapes_of(case)
    if case["op"] == "ortho":
        s["src"] = [gradient_like(g, r, c).to(DTYPES[case["dtype"]]) for r, c in shapes]
        s["dst"] = [torch.empty(r, c, device="cuda", dtype=DTYPES[case["out"]]) for r, c in shapes]
    else:
        s["grad"] = [gradient_like(g, r, c) for r, c in shapes]
        s["momentum_buffers"] = [gradient_like(g, r, c) * 5.0 for r, c in shapes]
        s["master"] = [torch.randn(r, c, generator=g, device="cuda") * 0.02 for r, c in shapes]
        s["copy"] = [w.to(torch.bfloat16) for w in s["master"]]
    return s


def run(s):
    return (own_form if own else plain_form)[s["op"]](s)


# ---- the framework's operators ----
def own_logprob(s):
    import paper_2401_15207_amd as H
    H.kernel_token_logprob(s["logits"], s["vocab"], s["targets"], s["scale"], s["logp"], s["entropy"], s["stats"], s["top_logp"], s["top_ids"])
    return {k: s[k] for k in ("logp", "entropy", "top_logp", "top_ids")}


def own_logprob_bwd(s):
    import paper_2401_15207_amd as H
    H.kernel_token_logprob_bwd(s["logits"], s["vocab"], s["targets"], s["scale"], s["stats"], s["entropy"], s["d_logp"], s["d_entropy"], s["dlogits"])
    return s["dlogits"][:, :s["vocab"]]


def own_ortho(s):
    import paper_2401_15207_amd as H
    H.kernel_orthogonalize(s["src"], s["dst"], steps=STEPS, coefficients=COEF, eps=EPS)
    return s["dst"]


def own_muon(s):
    import paper_2401_15207_amd as H
    H.kernel_muon(dict(kind="muon", lr=s["lr"], momentum=s["momentum"], weight_decay=s["decay"]), s["master"], s["grad"], s["momentum_buffers"], s["copy"])
    return {"master": s["master"], "momentum": s["momentum_buffers"], "copy": s["copy"]}


# ---- their plain forms ----
def plain_logprob(s):
    x = s["logits"][:, :s["vocab"]].float()
    z = x * s["scale"]
    z = z - z.max(1, keepdim=True).values
    e = torch.exp(z)
    total = e.sum(1)
    log_total = total.log()
    target = s["targets"].long()
    logp = torch.where(target < 0, 0.0, z.gather(1, target.clamp(min=0).unsqueeze(1)).squeeze(1) - log_total)
    entropy = log_total - torch.where(e > 0, e * z, 0.0).sum(1) / total
    ids = plain_top(x, s["top"]) if s["top"] else torch.empty(x.shape[0], 0, dtype=torch.long, device=x.device)
    return {"logp": logp, "entropy": entropy, "top_logp": z.gather(1, ids) - log_total.unsqueeze(1), "top_ids": ids.to(torch.int32)}


def plain_top(x, k):
    """Ids of the k largest, equal values in the order of their ids: value and id in one whole number."""
    bits = (x + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * 2 ** 32 + (2 ** 32 - 1 - torch.arange(x.shape[1], device=x.device))
    return 2 ** 32 - 1 - (torch.topk(order, k, dim=1).values & 0xFFFFFFFF)


def plain_logprob_bwd(s):
    logp = (s["logits"][:, :s["vocab"]].float() * s["scale"] - s["stats"][:, :1]) - s["stats"][:, 1:]
    p = torch.exp(logp)
    target = s["targets"].long().unsqueeze(1)
    g = torch.where(target < 0, 0.0, s["d_logp"].unsqueeze(1))
    d = -p * (g + s["d_entropy"].unsqueeze(1) * torch.where(p > 0, logp + s["entropy"].unsqueeze(1), 0.0))
    d.scatter_add_(1, target.clamp(min=0), g)
    return (d * s["scale"]).to(s["logits"].dtype)


def plain_newton_schulz(u):
    x = u.float()
    x = x / torch.sqrt((x * x).sum()).clamp(min=EPS)
    x = x.t() if u.shape[0] > u.shape[1] else x
    a, b, c = COEF
    for _ in range(STEPS):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.t() if u.shape[0] > u.shape[1] else x


def plain_ortho(s):
    return [plain_newton_schulz(u).to(d.dtype) for u, d in zip(s["src"], s["dst"])]


def plain_muon_one(s, w, g, m, copy):
    m.mul_(s["momentum"]).add_(g)
    step = plain_newton_schulz(g + s["momentum"] * m)
    w.copy_((1.0 - s["lr"] * s["decay"]) * w - s["lr"] * 0.2 * math.sqrt(max(w.shape)) * step)
    copy.copy_(w)


def plain_muon(s):
    [plain_muon_one(s, *each) for each in zip(s["master"], s["grad"], s["momentum_buffers"], s["copy"])]
    return {"master": s["master"], "momentum": s["momentum_buffers"], "copy": s["copy"]}


own_form = {"logprob": own_logprob, "logprob_bwd": own_logprob_bwd, "ortho": own_ortho, "muon": own_muon}
plain_form = {"logprob": plain_logprob, "logprob_bwd": plain_logprob_bwd, "ortho": plain_ortho, "muon": plain_muon}


def work(case):
    if case["op"].startswith("logprob"):
        rows, size = case["rows"], case["rows"] * case["vocab"] * (2 if case["dtype"] == "bf16" else 4)
        if case["op"] == "logprob":
            return {"bytes": size + rows * (4 + 8 + 8 + 8 * case["top"]), "flops": 6.0 * rows * case["vocab"]}
        return {"bytes": 2 * size + rows * 24, "flops": 8.0 * rows * case["vocab"]}
    total = {"bytes": 0.0, "flops": 0.0}
    for r, c in shapes_of(case):
        n, m = min(r, c), max(r, c)
        # the two symmetric products by half of their entries
        total["flops"] += STEPS * (1.0 * n * n * m + 1.0 * n ** 3 + 2.0 * n * n * m)
        if case["op"] == "ortho":
            total["bytes"] += r * c * ((2 if case["dtype"] == "bf16" else 4) + (2 if case["out"] == "bf16" else 4))
        else:
            total["bytes"] += r * c * 22.0
    return total


# ---- from the definitions, in 64 bits ----
def exact_orthogonal(u):
    """The odd polynomial of the singular values, applied on the shorter side: u q_1 q_2 ... with q_i = a + b t + c t^2 of t = x^T x (or x x^T)."""
    x = u.double()
    norm = torch.linalg.vector_norm(x).item()
    x = x / max(norm, EPS)
    a, b, c = COEF
    eye = torch.eye(min(u.shape), device=u.device, dtype=torch.float64)
    for _ in range(STEPS):
        if u.shape[0] > u.shape[1]:
            t = torch.mm(x.t().contiguous(), x)
            x = torch.mm(x, a * eye + torch.mm(t, b * eye + c * t))
        else:
            t = torch.mm(x, x.t().contiguous())
            x = torch.mm(a * eye + torch.mm(t, b * eye + c * t), x)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("logprob"):
        z = s["logits"][:, :case["vocab"]].double() / case["temperature"]
        lse = torch.logsumexp(z, 1, keepdim=True)
        logp = z - lse
        p = logp.exp()
        entropy = torch.special.entr(p).sum(1)
        target = s["targets"].long()
        has = target >= 0
        at = torch.arange(case["rows"], device=z.device)[has]
        if case["op"] == "logprob":
            chosen = torch.zeros(case["rows"], device=z.device, dtype=torch.float64)
            chosen[has] = logp[at, target[has]]
            # a double holds a logit and is sorted stably, so equal logits stay in the order of their ids
            ids = torch.sort(s["logits"][:, :case["vocab"]].double(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
            return {"logp": chosen, "entropy": entropy, "top_logp": logp.gather(1, ids), "top_ids": ids.to(torch.int32)}
        g = torch.where(has, s["d_logp"].double(), 0.0)
        # entropy's gradient: -p (ln p + H), and entr(p) = -p ln p
        d = -g.unsqueeze(1) * p + s["d_entropy"].double().unsqueeze(1) * (torch.special.entr(p) - p * entropy.unsqueeze(1))
        d[at, target[has]] += g[has]
        return d / case["temperature"]
    if case["op"] == "ortho":
        return [exact_orthogonal(u) for u in s["src"]]
    master, momentum = [], []
    for w, g, m in zip(s["master"], s["grad"], s["momentum_buffers"]):
        buf = case["momentum"] * m.double() + g.double()
        step = exact_orthogonal(g.double() + case["momentum"] * buf)
        w = w.double() * (1.0 - case["lr"] * case["decay"]) - case["lr"] * 0.2 * math.sqrt(max(w.shape)) * step
        master.append(w)
        momentum.append(buf)
    return {"master": master, "momentum": momentum, "copy": master}
