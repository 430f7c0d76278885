"""The operators of training and serving an exit head beyond its decision, with cases to time and check them.

Three of them, each in a plain form (elementary torch operations in 32 bits, 64 where a rounding border or a long sum
needs it) and as this package's calls:

  ce      the cross-entropy of a head over the whole vocabulary and its gradient with respect to the hidden states, the
          head's weights and its LayerNorm, without keeping the logits (ee_head_ce, ee_head_ce_grad)
  q4      a head whose weights are held in 4 bits with a scale per group of columns: writing them, reading them back,
          and the exit decision from them (ee_head_q4_pack, ee_head_q4_unpack, ee_exit_head_q4)
  embed   the scaled embedding lookup that shares its table with the head, and its gradient (ee_embed, ee_embed_grad)
"""
import math

import torch

own = False

LN_EPS = 1e-5
V_PYTHIA = 50304


def listed():
    return [
        # evaluating one head's loss on a held-out slice: the smallest cross-entropy call, one read of the weights
        {"name": "ce_eval_64", "op": "ce", "form": "eval", "M": 64, "d": 512, "V": V_PYTHIA, "ignored": 0.0},
        # a training step of one head on a batch of ordinary length
        {"name": "ce_step_4096", "op": "ce", "form": "step", "M": 4096, "d": 1024, "V": V_PYTHIA, "ignored": 0.0},
        # a padded batch of odd length with a vocabulary that fits no tile
        {"name": "ce_step_ragged", "op": "ce", "form": "step", "M": 1003, "d": 520, "V": 32003, "ignored": 0.3},
        # a training step over the largest batch and width the heads are used with
        {"name": "ce_step_16384", "op": "ce", "form": "step", "M": 16384, "d": 2560, "V": V_PYTHIA, "ignored": 0.05},
        # drafting: one token
        {"name": "q4_head_1", "op": "q4", "form": "head", "M": 1, "d": 1024, "V": V_PYTHIA, "group": 64},
        # drafting: a small batch on the smallest model's head
        {"name": "q4_head_8", "op": "q4", "form": "head", "M": 8, "d": 512, "V": V_PYTHIA, "group": 32},
        # a decoding batch
        {"name": "q4_head_64", "op": "q4", "form": "head", "M": 64, "d": 1024, "V": V_PYTHIA, "group": 64},
        # a batch of odd size on a wide head with an odd vocabulary
        {"name": "q4_head_33", "op": "q4", "form": "head", "M": 33, "d": 2560, "V": 50257, "group": 128},
        # writing a trained head in 4 bits, and what those bits stand for
        {"name": "q4_pack_2048", "op": "q4", "form": "pack", "M": 0, "d": 2048, "V": V_PYTHIA, "group": 64},
        # the tokens of one drafting step
        {"name": "embed_32", "op": "embed", "form": "lookup", "n": 32, "d": 1024, "V": V_PYTHIA, "wide": False},
        # a training batch's gradient into the table, tokens as frequent as in text
        {"name": "embed_grad_16384", "op": "embed", "form": "grad", "n": 16384, "d": 1024, "V": V_PYTHIA, "wide": False},
        # a short batch's gradient, kept in 32 bits
        {"name": "embed_grad_257", "op": "embed", "form": "grad", "n": 257, "d": 520, "V": 32003, "wide": True},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ce", "ce", "q4", "q4", "embed"])
    d = 8 * _spread(rng, 8, 320)
    V = _spread(rng, 1000, 60000)
    if op == "ce":
        return {"op": "ce", "form": rng.choice(["eval", "step", "step"]), "M": _spread(rng, 1, 12000), "d": d, "V": V,
                "ignored": rng.choice([0.0, 0.1, 0.5])}
    if op == "q4":
        form = rng.choice(["head", "head", "head", "pack"])
        group = rng.choice([32, 64, 128])
        return {"op": "q4", "form": form, "M": _spread(rng, 1, 100) if form == "head" else 0, "d": group * max(1, d // group), "V": V,
                "group": group}
    return {"op": "embed", "form": rng.choice(["lookup", "grad"]), "n": _spread(rng, 1, 40000), "d": d, "V": V, "wide": rng.random() < 0.5}


def _bf16(x):
    return x.to(torch.bfloat16)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 1000003 + 17)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=dev)

    d, V = case["d"], case["V"]
    s = dict(case)
    W = _bf16(0.02 * normal(V, d))
    if case["op"] == "embed":
        n = case["n"]
        # log-uniform ranks: the most frequent token takes several per cent of the batch, most rows of the table none
        rank = torch.exp(uniform(n) * math.log(V)).to(torch.int64).sub_(1).clamp_(0, V - 1)
        s["tokens"] = torch.randperm(V, generator=gen, device=dev)[rank].to(torch.int32)
        s["scale"] = math.sqrt(d)
        if case["form"] == "lookup":
            s["table"] = W
        else:
            s["dout"] = _bf16(normal(n, d) / math.sqrt(n))
        if own and case["form"] == "grad":
            import paper_2407_21082_b200 as ee
            s["workspace"] = ee.new_embed_grad_workspace(n, d, V)
        return s
    if case["form"] == "pack":
        s["W"] = W
        return s
    # hidden rows that lean towards the weight row of one token each, from hardly to strongly, as a model's do: that token's
    # logit comes to about 0 .. 15, against about ln V for all the others together
    M = case["M"]
    target = torch.randint(0, V, (M,), generator=gen, device=dev)
    w = W[target].float()
    w = w / w.norm(dim=1, keepdim=True)
    logit = 7.0 + 9.0 * uniform(M, 1) if case["op"] == "q4" else 14.0 * uniform(M, 1)
    lean = (logit / (0.02 * d)).clamp(max=0.95)
    h = (1 - lean * lean).sqrt() * normal(M, d) + lean * math.sqrt(d) * w
    s["h"] = _bf16(2.0 * h + 0.1)
    s["gamma"] = 1.0 + 0.1 * normal(d)
    s["beta"] = 0.02 * normal(d)
    if case["op"] == "ce":
        s["W"] = W
        other = torch.randint(0, V, (M,), generator=gen, device=dev)
        labels = torch.where(uniform(M) < 0.8, target, other)
        s["labels"] = torch.where(uniform(M) < case["ignored"], torch.full_like(labels, -1), labels).to(torch.int32)
        if own:
            import paper_2407_21082_b200 as ee
            s["workspace"] = ee.new_head_ce_workspace(M, d, V) if case["form"] == "eval" else ee.new_head_ce_grad_workspace(M, d, V)
        return s
    s["tau"] = 2.0
    s["q"], s["scales"] = _quantise(W, case["group"])
    if own:       # the same weights as a serving program holds them: packed once, when they are loaded
        import paper_2407_21082_b200 as ee
        s["weights"] = ee.ee_head_q4_pack(W, case["group"])
        s["workspace"] = ee.new_exit_head_q4_workspace(M, s["weights"])
    return s


# ---------------------------------------------------------------- plain forms

def _layer_norm(h, gamma, beta):
    """y rounded to bf16 as the heads define it (64 bits before the rounding: a value next to a border), and what the backward needs."""
    x = h.double()
    mu = x.mean(dim=1, keepdim=True)
    rstd = torch.rsqrt(((x - mu) ** 2).mean(dim=1, keepdim=True) + LN_EPS)
    xhat = (x - mu) * rstd
    y = _bf16(xhat * gamma.double() + beta.double())
    return y.float(), xhat.float(), rstd.float()


def _quantise(W, group):
    """Whole numbers -8 .. 7 and one bf16 scale per row and group of columns: a seventh of the group's largest magnitude."""
    V, d = W.shape
    w = W.float().view(V, d // group, group)
    scales = _bf16(w.abs().amax(dim=2) / 7.0)
    s = scales.float().unsqueeze(2)
    q = torch.where(s > 0, torch.round(w / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(w)).clamp(-8, 7)
    return q.to(torch.int8).view(V, d), scales


def _values(q, scales):
    """What the whole numbers and scales stand for: the product, rounded once to bf16."""
    V, d = q.shape
    return _bf16(q.view(V, scales.shape[1], -1).float() * scales.float().unsqueeze(2)).view(V, d)


def _plain_ce(s):
    labels, V = s["labels"].long(), s["V"]
    y, xhat, rstd = _layer_norm(s["h"], s["gamma"], s["beta"])
    Wf = s["W"].float()
    z = y @ Wf.t()
    lse = torch.logsumexp(z, dim=1)
    counted = (labels >= 0) & (labels < V)
    at = torch.where(counted, labels, torch.zeros_like(labels)).unsqueeze(1)
    ce = torch.where(counted, lse - z.gather(1, at).squeeze(1), torch.zeros_like(lse))
    n = counted.sum()
    loss = torch.stack([(ce.double().sum() / n.clamp(min=1)).float(), n.float()])
    out = {"ce": ce, "lse": lse, "loss": loss}
    if s["form"] == "eval":
        return out
    g = torch.exp(z - lse.unsqueeze(1))
    g.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    g *= (counted.float() / n.clamp(min=1)).unsqueeze(1)
    dy = g @ Wf
    dW = g.t() @ y
    t = dy * s["gamma"]
    dh = rstd * (t - t.mean(dim=1, keepdim=True) - xhat * (t * xhat).mean(dim=1, keepdim=True))
    out.update(dh=_bf16(dh), dW=_bf16(dW), dgamma=_bf16((dy * xhat).sum(dim=0)), dbeta=_bf16(dy.sum(dim=0)))
    return out


def _plain_head(s):
    y, _, _ = _layer_norm(s["h"], s["gamma"], s["beta"])
    z = y @ _values(s["q"], s["scales"]).float().t()
    m, argmax = z.max(dim=1)
    argmax = torch.where(z == m.unsqueeze(1), torch.arange(s["V"], device=z.device), s["V"]).amin(dim=1)
    e = torch.exp(z - m.unsqueeze(1))
    total = e.sum(dim=1)
    entropy = torch.log(total) - (e * (z - m.unsqueeze(1))).sum(dim=1) / total
    return {"argmax": argmax.to(torch.int32), "entropy": entropy, "maxprob": 1.0 / total, "exit_mask": (entropy < s["tau"]).to(torch.uint8)}


def _plain_embed(s):
    if s["form"] == "lookup":
        return _bf16(s["table"][s["tokens"].long()].float() * s["scale"])
    out = torch.zeros(s["V"], s["d"], device=s["dout"].device)
    out.index_add_(0, s["tokens"].long(), s["dout"].float())
    out *= s["scale"]
    return out if s["wide"] else _bf16(out)


# ---------------------------------------------------------------- one pass

def run(state):
    s = state
    if own:
        return _own(s)
    if s["op"] == "ce":
        return _plain_ce(s)
    if s["op"] == "embed":
        return _plain_embed(s)
    if s["form"] == "pack":
        return _values(*_quantise(s["W"], s["group"]))
    return _plain_head(s)


def _own(s):
    import paper_2407_21082_b200 as ee
    if s["op"] == "ce":
        head = dict(h=s["h"], gamma=s["gamma"], beta=s["beta"], W=s["W"])
        out = dict(ee.ee_head_ce(head, s["labels"], LN_EPS, workspace=s["workspace"]))
        if s["form"] == "step":
            out.update(ee.ee_head_ce_grad(head, s["labels"], LN_EPS, out, workspace=s["workspace"]))
        return out
    if s["op"] == "embed":
        if s["form"] == "lookup":
            return ee.ee_embed(s["table"], s["tokens"], s["scale"])
        return ee.ee_embed_grad(s["dout"], s["tokens"], s["V"], s["scale"], dtype=torch.float32 if s["wide"] else torch.bfloat16,
                                workspace=s["workspace"])
    if s["form"] == "pack":
        return ee.ee_head_q4_unpack(ee.ee_head_q4_pack(s["W"], s["group"]))
    return ee.ee_exit_head_q4(s["h"], s["gamma"], s["beta"], LN_EPS, s["weights"], s["tau"], workspace=s["workspace"])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    d, V = case["d"], case["V"]
    if case["op"] == "embed":
        n = case["n"]
        if case["form"] == "lookup":
            return {"bytes": n * d * 4 + n * 4, "flops": n * d}
        return {"bytes": n * d * 2 + n * 4 + V * d * (4 if case["wide"] else 2), "flops": n * d}
    if case["form"] == "pack":
        packed = V * d // 2 + V * (d // case["group"]) * 2
        return {"bytes": V * d * 2 + 2 * packed + V * d * 2, "flops": 2 * V * d}
    M = case["M"]
    if case["op"] == "q4":
        return {"bytes": V * d // 2 + V * (d // case["group"]) * 2 + M * d * 2 + M * 13, "flops": 2 * M * V * d}
    b = M * d * 2 + V * d * 2 + M * 4 + M * 8
    if case["form"] == "eval":
        return {"bytes": b, "flops": 2 * M * V * d}
    return {"bytes": b + M * d * 2 + V * d * 2 + d * 4, "flops": 6 * M * V * d}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_rows(h, gamma, beta):
    x = h.to(torch.float64)
    c = x - x.sum(dim=1, keepdim=True) / x.shape[1]
    rstd = 1.0 / torch.sqrt((c * c).sum(dim=1, keepdim=True) / x.shape[1] + LN_EPS)
    return (c * rstd * gamma.to(torch.float64) + beta.to(torch.float64)).to(torch.bfloat16).to(torch.float64), c * rstd, rstd


def _exact_ce(case, s):
    y, xhat, rstd = _exact_rows(s["h"], s["gamma"], s["beta"])
    W = s["W"].to(torch.float64)
    M, V = case["M"], case["V"]
    ce = torch.zeros(M, dtype=torch.float64, device=W.device)
    lse = torch.empty_like(ce)
    dy = torch.zeros_like(y)
    dW = torch.zeros_like(W)
    counted = s["labels"] >= 0
    n = int(counted.sum())
    for r in range(0, M, 2048):          # blocks of rows: the logits of one block at a time
        rows = slice(r, min(r + 2048, M))
        p = y[rows] @ W.t()
        top = p.amax(dim=1, keepdim=True)
        lse[rows] = top[:, 0] + torch.log(torch.exp(p - top).sum(dim=1))
        k = torch.nonzero(counted[rows])[:, 0]
        lab = s["labels"][rows][k].long()
        ce[r + k] = lse[rows][k] - p[k, lab]
        if case["form"] == "step":
            p = torch.exp(p - lse[rows].unsqueeze(1))
            p[k, lab] -= 1.0
            p *= (counted[rows].to(torch.float64) / max(n, 1)).unsqueeze(1)
            dy[rows] = p @ W
            dW += p.t() @ y[rows]
        del p
    out = {"ce": ce, "lse": lse, "loss": torch.stack([ce.sum() / max(n, 1), torch.tensor(float(n), dtype=torch.float64, device=W.device)])}
    if case["form"] == "step":
        t = dy * s["gamma"].to(torch.float64)
        dh = rstd * (t - t.sum(dim=1, keepdim=True) / t.shape[1] - xhat * ((t * xhat).sum(dim=1, keepdim=True) / t.shape[1]))
        out.update(dh=dh, dW=dW, dgamma=(dy * xhat).sum(dim=0), dbeta=dy.sum(dim=0))
    return out


def _exact_weights(W, group):
    """Values of the 4-bit form, from the definition: nearest whole number of scales, ties to the even one."""
    V, d = W.shape
    w = W.to(torch.float64).reshape(V, d // group, group)
    scale = (w.abs().max(dim=2, keepdim=True).values / 7.0).to(torch.float32).to(torch.bfloat16).to(torch.float64)
    q = torch.round(w / scale.clamp(min=1e-300)).clamp(-8, 7)
    q = torch.where(scale > 0, q, torch.zeros_like(q))
    return (q * scale).to(torch.bfloat16).to(torch.float64).reshape(V, d)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "ce":
        return _exact_ce(case, s)
    if case["op"] == "embed":
        if case["form"] == "lookup":
            return s["table"].to(torch.float64)[s["tokens"].long()] * s["scale"]
        out = torch.zeros(case["V"], case["d"], dtype=torch.float64, device=s["dout"].device)
        return out.index_put_((s["tokens"].long(),), s["dout"].to(torch.float64) * s["scale"], accumulate=True)
    if case["form"] == "pack":
        return _exact_weights(s["W"], case["group"])
    # the whole numbers and scales are inputs here
    V, d, g = case["V"], case["d"], case["group"]
    W = (s["q"].to(torch.float64).reshape(V, d // g, g) * s["scales"].to(torch.float64)[:, :, None]).to(torch.bfloat16).to(torch.float64)
    y, _, _ = _exact_rows(s["h"], s["gamma"], s["beta"])
    z = y @ W.reshape(V, d).t()
    z = z - z.max(dim=1, keepdim=True).values
    total = torch.exp(z).sum(dim=1)
    entropy = torch.log(total) - (torch.exp(z) * z).sum(dim=1) / total
    return {"argmax": None, "entropy": entropy, "maxprob": 1.0 / total, "exit_mask": None}
