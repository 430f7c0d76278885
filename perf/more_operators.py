"""The operators of improving a head by what it drafted, and of drafting from 4-bit floating point, with cases to time and check them.

Each in a plain form (elementary torch operations in 32 bits, 64 where a border or a long sum needs it) and as this package's calls:

  policy      the clipped policy loss over drafted tokens with a penalty for leaving a reference head, and its gradient with
              respect to the tokens' cross-entropies, which ee_head_ce_grad takes as weights (ee_policy_loss)
  preference  the loss of pairs of sequences, one preferred to the other, and the same gradient (ee_preference_loss)
  clip        the norm over all of a step's gradients, and their scaling where it is too large (ee_grad_clip, GradClip)
  fp4         a head held in microscaled 4-bit floating point: writing and reading it (ee_head_fp4_pack, ee_head_fp4_unpack), and
              the exit decision from it with activations in the same form (ee_exit_head_fp4)
"""
import math

import torch

own = False

LN_EPS = 1e-5
V_PYTHIA = 50304
CLIP_LOW, CLIP_HIGH = 0.2, 0.28


def listed():
    return [
        # the tokens of one drafting batch: the smallest loss, all latency
        {"name": "policy_512", "op": "policy", "tokens": 512, "seqs": 16, "mean": "token", "kl": 0.0},
        # a step over a batch of ragged answers, each answer counting the same
        {"name": "policy_65537", "op": "policy", "tokens": 65537, "seqs": 200, "mean": "sequence", "kl": 0.04},
        # eight pairs of short answers
        {"name": "preference_8", "op": "preference", "tokens": 4001, "pairs": 8, "reference": True},
        # few pairs of long documents: a long axis and hardly any rows
        {"name": "preference_long", "op": "preference", "tokens": 300000, "pairs": 3, "reference": True},
        # the LayerNorm parameters' gradients of a few heads
        {"name": "clip_small", "op": "clip", "V": 1, "d": 1024, "heads": 4, "extra": 0, "table": False},
        # what a training step of one head leaves: its weights' gradient and its LayerNorm's
        {"name": "clip_head", "op": "clip", "V": V_PYTHIA, "d": 1024, "heads": 1, "extra": 0, "table": False},
        # three wide heads, adapters of odd sizes in 16 and 32 bits, and a table's gradient kept in 32 bits
        {"name": "clip_many", "op": "clip", "V": 32003, "d": 2560, "heads": 3, "extra": 40, "table": True},
        # drafting: one token
        {"name": "fp4_head_1", "op": "fp4", "form": "head", "M": 1, "d": 1024, "V": V_PYTHIA, "group": 16},
        # a decoding batch on the smallest model's head
        {"name": "fp4_head_64", "op": "fp4", "form": "head", "M": 64, "d": 512, "V": V_PYTHIA, "group": 32},
        # a verification pass of odd size with a vocabulary and a width that fit no tile
        {"name": "fp4_head_ragged", "op": "fp4", "form": "head", "M": 203, "d": 1056, "V": 50257, "group": 32},
        # the largest batch and width the heads are used with
        {"name": "fp4_head_16384", "op": "fp4", "form": "head", "M": 16384, "d": 2560, "V": V_PYTHIA, "group": 16},
        # writing a trained head in 4 bits, and what those bits stand for
        {"name": "fp4_pack_2048", "op": "fp4", "form": "pack", "M": 0, "d": 2048, "V": V_PYTHIA, "group": 16},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["policy", "preference", "clip", "fp4", "fp4"])
    if op == "policy":
        tokens = _spread(rng, 100, 300000)
        return {"op": op, "tokens": tokens, "seqs": _spread(rng, 1, max(2, tokens // 16)), "mean": rng.choice(["token", "sequence"]),
                "kl": rng.choice([0.0, 0.04])}
    if op == "preference":
        tokens = _spread(rng, 100, 300000)
        return {"op": op, "tokens": tokens, "pairs": _spread(rng, 1, max(2, tokens // 32)), "reference": rng.random() < 0.7}
    if op == "clip":
        return {"op": op, "V": _spread(rng, 1, 32003), "d": 8 * _spread(rng, 32, 320), "heads": rng.randint(1, 3), "extra": rng.choice([0, 0, 7, 40]),
                "table": rng.random() < 0.3}
    form = rng.choice(["head", "head", "head", "pack"])
    return {"op": op, "form": form, "M": _spread(rng, 1, 12000) if form == "head" else 0, "d": 32 * _spread(rng, 8, 80),
            "V": _spread(rng, 8000, 60000), "group": rng.choice([16, 32])}


def _bf16(x):
    return x.to(torch.bfloat16)


def _boundaries(total, n, uniform):
    """n + 1 boundaries of ragged sequences that fill `total` tokens; some may be empty."""
    cuts = torch.sort((uniform(n - 1) * (total + 1)).to(torch.int64).clamp_(0, total))[0]
    ends = cuts.new_tensor([0, total])
    return torch.cat([ends[:1], cuts, ends[1:]]).to(torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 1000003 + 29)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=dev)

    s = dict(case)
    op = case["op"]
    if op in ("policy", "preference"):
        n = case["tokens"]
        # what heads' losses look like: most tokens nearly certain, some hard; the head has moved a little from the one that drafted
        # and somewhat more from the reference
        s["ce"] = -torch.log1p(-0.999 * uniform(n)) * torch.exp(normal(n))
        s["V"] = V_PYTHIA
        labels = torch.randint(0, V_PYTHIA, (n,), generator=gen, device=dev)
        s["labels"] = torch.where(uniform(n) < 0.25, torch.full_like(labels, -1), labels).to(torch.int32)      # prompts and padding
        s["ref_ce"] = (s["ce"] + 0.3 * normal(n)).abs()
        counted = (s["labels"] >= 0).sum()
        s["counted"] = torch.stack([(s["ce"] * (s["labels"] >= 0)).sum() / counted.clamp(min=1), counted]).float()       # as ee_head_ce leaves it
        if op == "policy":
            s["old_ce"] = (s["ce"] + 0.15 * normal(n)).abs()
            by_sequence = case["mean"] == "sequence"
            s["seq_start"] = _boundaries(n, case["seqs"], uniform) if by_sequence else None
            s["adv"] = normal(case["seqs"] if by_sequence else n)
        else:
            s["seq_start"] = _boundaries(n, 2 * case["pairs"], uniform)
            s["beta"], s["smoothing"] = 0.1, 0.05
        if own:
            import paper_2407_21082_b200 as ee
            s["workspace"] = ee.new_token_loss_workspace()
            s["out"] = ee.new_policy_loss_outputs(n) if op == "policy" else ee.new_preference_loss_outputs(n, case["pairs"])
        return s
    V, d = case["V"], case["d"]
    if op == "clip":
        grads = []
        for _ in range(case["heads"]):
            grads += [_bf16(1e-3 * normal(V, d)), _bf16(1e-2 * normal(d)), _bf16(1e-2 * normal(d))]
        for i in range(case["extra"]):
            n = 1 + (i * 7919) % 49999
            grads.append(1e-2 * normal(n) if i % 3 == 0 else _bf16(1e-2 * normal(n)) if i % 3 == 1 else (1e-2 * normal(n)).half())
        if case["table"]:
            grads.append(1e-3 * normal(V, d) * (uniform(V, 1) < 0.2))                    # most tokens do not occur in a batch
        s["grads"] = grads
        s["max_norm"] = 1.0 if V * d > 3000000 else 0.25
        if own:       # a training program's gradient buffers are the same from step to step: their list is made once
            import paper_2407_21082_b200 as ee
            s["clip"] = ee.GradClip(grads, out=[torch.empty_like(g) for g in grads])
        return s
    spread = max(0.02, 20.0 / d)
    W = _bf16(spread * normal(V, d))
    if case["form"] == "pack":
        s["W"] = W
        return s
    # hidden rows that lean towards the weight row of one token each: most so much that the head is nearly sure of it, the others
    # so little that it is lost, as a model's do
    M = case["M"]
    target = torch.randint(0, V, (M,), generator=gen, device=dev)
    w = W[target].float()
    w = w / w.norm(dim=1, keepdim=True)
    others = math.log(V) + spread * spread * d / 2
    logit = torch.where(uniform(M, 1) < 0.7, others + 2.5 + 4.5 * uniform(M, 1), others - 2.2 - uniform(M, 1))
    lean = (logit / (spread * d)).clamp(max=0.97)
    s["h"] = _bf16(2.0 * ((1 - lean * lean).sqrt() * normal(M, d) + lean * math.sqrt(d) * w) + 0.1)
    s["gamma"] = 1.0 + 0.1 * normal(d)
    s["beta"] = 0.02 * normal(d)
    s["tau"] = 3.0
    s["q"], s["scales"] = _quantise(W, case["group"], False)
    if own:       # the same weights as a serving program holds them: packed once, when they are loaded
        import paper_2407_21082_b200 as ee
        s["weights"] = ee.ee_head_fp4_pack(W, case["group"])
        s["workspace"], s["out"] = ee.new_exit_head_fp4_workspace(M, s["weights"]), ee.new_outputs(M)
    return s


# ---------------------------------------------------------------- plain forms

def _exponent(x):
    """floor(log2 x) of positive x, -1000 of 0."""
    e = torch.frexp(x)[1] - 1
    return torch.where(x > 0, e, torch.full_like(e, -1000))


def _two_to(e):
    return torch.exp2(e.double())


def _quantise(x, group, by_row):
    """Numbers of 4 bits (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and what a group of them is multiplied with.  Groups of 32 have a
    power of two; groups of 16 a number of 8 bits (four of exponent, three of mantissa) times a power of two that all of x
    (by_row: each of its rows) has in common.  In 64 bits, where all of it is exact up to the roundings that are meant."""
    n, d = x.shape
    v = x.float().view(n, d // group, group)
    top = v.abs().amax(dim=2)
    if group == 32:
        scale = _two_to((_exponent(top) - 2).clamp(-127, 127))
    else:
        highest = top.amax(dim=1, keepdim=True) if by_row else top.amax()
        common = _two_to(torch.where(highest > 0, (_exponent(highest) - 10).clamp(min=-126), torch.zeros_like(_exponent(highest))))
        scale = (top.double() / common / 6.0).float().to(torch.float8_e4m3fn).double() * common
    a = v.double() / torch.where(scale > 0, scale, torch.ones_like(scale)).unsqueeze(2)
    m = a.abs()
    m = torch.where(m < 2, torch.round(2 * m) / 2, torch.where(m < 4, torch.round(m), 2 * torch.round(m / 2))).clamp(max=6)
    q = torch.where((scale > 0).unsqueeze(2), torch.copysign(m, a), torch.zeros_like(m))
    return q.float().to(torch.bfloat16).view(n, d), scale.float()


def _values(q, scales):
    n, d = q.shape
    return (q.float().view(n, scales.shape[1], -1) * scales.unsqueeze(2)).view(n, d)


def _layer_norm(h, gamma, beta):
    """Rounded to bf16 as the heads define it; 64 bits before, for values next to a border."""
    x = h.double()
    mu = x.mean(dim=1, keepdim=True)
    rstd = torch.rsqrt(((x - mu) ** 2).mean(dim=1, keepdim=True) + LN_EPS)
    return _bf16(((x - mu) * rstd * gamma.double() + beta.double()).float())


def _plain_head(s):
    y = _values(*_quantise(_layer_norm(s["h"], s["gamma"], s["beta"]), s["group"], True))
    z = y @ _values(s["q"], s["scales"]).t()
    m, argmax = z.max(dim=1)
    argmax = torch.where(z == m.unsqueeze(1), torch.arange(s["V"], device=z.device), s["V"]).amin(dim=1)
    z = z - m.unsqueeze(1)
    e = torch.exp(z)
    # without the largest term, beside which the digits of a nearly certain row's others would be lost
    e.scatter_(1, argmax.unsqueeze(1), 0.0)
    rest = e.sum(dim=1)
    entropy = torch.log1p(rest) - (e * z).sum(dim=1) / (1.0 + rest)
    return {"argmax": argmax.to(torch.int32), "entropy": entropy, "maxprob": 1.0 / (1.0 + rest), "exit_mask": (entropy < s["tau"]).to(torch.uint8)}


def _segments(s):
    """The sequence of each token and the number of sequences."""
    lengths = (s["seq_start"][1:] - s["seq_start"][:-1]).long()
    n = lengths.numel()
    return torch.repeat_interleave(torch.arange(n, device=lengths.device), lengths, output_size=s["tokens"]), n


def _plain_policy(s):
    counted = (s["labels"] >= 0) & (s["labels"] < s["V"])
    zero = torch.zeros((), dtype=torch.float64, device=counted.device)
    adv = s["adv"]
    if s["seq_start"] is None:
        weight = counted.double() / s["counted"][1].double().clamp(min=1)
    else:
        seq, n = _segments(s)
        have = torch.zeros(n, dtype=torch.float64, device=seq.device).index_add_(0, seq, counted.double())
        weight = counted.double() / (have.clamp(min=1) * n)[seq]
        adv = adv[seq]
    log_ratio = s["old_ce"].double() - s["ce"].double()
    ratio = torch.exp(log_ratio)
    adv = adv.double()
    cut = torch.where(adv > 0, log_ratio > math.log1p(CLIP_HIGH), (log_ratio < math.log1p(-CLIP_LOW)) & (adv < 0))
    held = torch.where(adv > 0, torch.full_like(ratio, 1.0 + CLIP_HIGH), torch.full_like(ratio, 1.0 - CLIP_LOW))
    policy = -adv * torch.where(cut, held, ratio)
    grad = torch.where(cut, zero, adv * ratio)
    kl = zero.expand_as(ratio)
    if s["kl"] > 0:
        gap = s["ce"].double() - s["ref_ce"].double()
        kl = torch.expm1(gap) - gap
        grad = grad + s["kl"] * torch.expm1(gap)

    def mean(x):
        return torch.where(counted, weight * x, zero).sum()

    loss = torch.stack([mean(policy + s["kl"] * kl), mean(policy), mean(kl), mean(cut.double())])
    return {"loss": loss.float(), "dce": torch.where(counted, weight * grad, zero).float()}


def _plain_preference(s):
    counted = (s["labels"] >= 0) & (s["labels"] < s["V"])
    seq, n = _segments(s)
    gain = -s["ce"].double()
    if s["reference"]:
        gain = gain + s["ref_ce"].double()
    gain = torch.where(counted, gain, torch.zeros_like(gain))
    reward = s["beta"] * torch.zeros(n, dtype=torch.float64, device=seq.device).index_add_(0, seq, gain)
    margin = reward[0::2] - reward[1::2]
    soft = s["smoothing"]
    loss = -((1 - soft) * torch.nn.functional.logsigmoid(margin) + soft * torch.nn.functional.logsigmoid(-margin))
    slope = (soft * torch.sigmoid(margin) - (1 - soft) * torch.sigmoid(-margin)) / margin.numel()
    side = torch.stack([-slope, slope], dim=1).view(-1) * s["beta"]
    dce = torch.where(counted, side[seq], torch.zeros_like(gain))
    means = torch.stack([loss.mean(), (margin > 0).double().mean(), reward[0::2].mean(), reward[1::2].mean()])
    return {"loss": means.float(), "margin": margin.float(), "dce": dce.float()}


def _plain_clip(s):
    total = torch.stack([(g.float() ** 2).sum(dtype=torch.float64) for g in s["grads"]]).sum()
    norm = torch.sqrt(total).float()
    factor = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0)
    return {"norm": norm.view(1), "grads": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


# ---------------------------------------------------------------- one pass

def run(state):
    s = state
    if own:
        return _own(s)
    if s["op"] == "policy":
        return _plain_policy(s)
    if s["op"] == "preference":
        return _plain_preference(s)
    if s["op"] == "clip":
        return _plain_clip(s)
    if s["form"] == "pack":
        return _bf16(_values(*_quantise(s["W"], s["group"], False)))
    return _plain_head(s)


def _own(s):
    import paper_2407_21082_b200 as ee
    if s["op"] == "policy":
        forward = {"ce": s["ce"], "loss": s["counted"]}
        return ee.ee_policy_loss(forward, s["labels"], s["V"], s["old_ce"], s["adv"], ref_ce=s["ref_ce"] if s["kl"] > 0 else None, kl_weight=s["kl"],
                                 clip=(CLIP_LOW, CLIP_HIGH), seq_start=s["seq_start"], out=s["out"], workspace=s["workspace"])
    if s["op"] == "preference":
        forward = {"ce": s["ce"], "loss": s["counted"]}
        return ee.ee_preference_loss(forward, s["labels"], s["V"], s["seq_start"], ref_ce=s["ref_ce"] if s["reference"] else None, beta=s["beta"],
                                     smoothing=s["smoothing"], out=s["out"], workspace=s["workspace"])
    if s["op"] == "clip":
        # into other buffers, so that the state's gradients stay what they are from pass to pass
        return {"norm": s["clip"](s["max_norm"]), "grads": s["clip"].out}
    if s["form"] == "pack":
        return ee.ee_head_fp4_unpack(ee.ee_head_fp4_pack(s["W"], s["group"]))
    return ee.ee_exit_head_fp4(s["h"], s["gamma"], s["beta"], LN_EPS, s["weights"], s["tau"], out=s["out"], workspace=s["workspace"])


# ---------------------------------------------------------------- what a pass cannot do without

def _clip_bytes(case):
    V, d = case["V"], case["d"]
    b = case["heads"] * (V * d + 2 * d) * 2 + (V * d * 4 if case["table"] else 0)
    return b + sum((1 + (i * 7919) % 49999) * (4 if i % 3 == 0 else 2) for i in range(case["extra"]))


def work(case):
    op = case["op"]
    if op == "policy":
        n, by_sequence = case["tokens"], case["mean"] == "sequence"
        return {"bytes": n * (16 + (4 if case["kl"] > 0 else 0) + (0 if by_sequence else 4)) + (case["seqs"] * 8 if by_sequence else 0), "flops": 20 * n}
    if op == "preference":
        return {"bytes": case["tokens"] * (12 + (4 if case["reference"] else 0)) + case["pairs"] * 12, "flops": 4 * case["tokens"]}
    if op == "clip":
        return {"bytes": 2 * _clip_bytes(case), "flops": 2 * _clip_bytes(case)}
    V, d, M = case["V"], case["d"], case["M"]
    packed = V * d // 2 + V * (d // case["group"])
    if case["form"] == "pack":
        return {"bytes": V * d * 2 + 2 * packed + V * d * 2, "flops": 2 * V * d}
    return {"bytes": packed + M * d * 2 + M * 13, "flops": 2 * M * V * d}


# ---------------------------------------------------------------- the definitions in 64 bits

_LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_four_bits(a):
    """Nearest level; of two equally near the one with the even number, which is the lower one at every second border."""
    out = torch.zeros_like(a)
    for i in range(1, 8):
        border = (_LEVELS[i - 1] + _LEVELS[i]) / 2
        reached = a.abs() > border if i % 2 == 1 else a.abs() >= border
        out = torch.where(reached, torch.full_like(out, _LEVELS[i]), out)
    return out * torch.sign(a)


def _exact_eight_bits(a):
    """Nearest number m 2^e with three bits behind the point of m and e >= -6, ties to the even m."""
    e = torch.floor(torch.log2(a.clamp(min=1e-300)))
    e = torch.where(torch.exp2(e) > a, e - 1, torch.where(torch.exp2(e + 1) <= a, e + 1, e)).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(a / step) * step


def _exact_values(x, group, by_row):
    v = x.to(torch.float64).reshape(x.shape[0], -1, group)
    top = v.abs().max(dim=2, keepdim=True).values
    power = torch.full_like(top, -1.0)

    def floor_log2(t):
        e = torch.floor(torch.log2(t.clamp(min=1e-300)))
        return torch.where(torch.exp2(e) > t, e - 1, torch.where(torch.exp2(e + 1) <= t, e + 1, e))

    if group == 32:
        scale = torch.exp2(floor_log2(top).sub_(2).clamp_(-127, 127))
    else:
        most = top.amax(dim=(1, 2), keepdim=True) if by_row else top.max().reshape(1, 1, 1)
        power = torch.where(most > 0, torch.exp2(floor_log2(most).sub_(10).clamp_(min=-126)), torch.ones_like(most))
        scale = _exact_eight_bits(top / (6.0 * power)) * power
    q = torch.where(scale > 0, _exact_four_bits(v / scale.clamp(min=1e-300)), torch.zeros_like(v))
    return (q * scale).reshape(x.shape)


def _exact_head(case, s):
    W = (s["q"].to(torch.float64).reshape(case["V"], -1, case["group"]) * s["scales"].to(torch.float64)[:, :, None]).reshape(case["V"], case["d"])
    entropy, maxprob = [], []
    for r in range(0, case["M"], 2048):          # blocks of rows: the logits of one block at a time
        x = s["h"][r:r + 2048].to(torch.float64)
        c = x - x.sum(dim=1, keepdim=True) / x.shape[1]
        y = c / torch.sqrt((c * c).sum(dim=1, keepdim=True) / x.shape[1] + LN_EPS) * s["gamma"].to(torch.float64) + s["beta"].to(torch.float64)
        y = _exact_values(y.to(torch.float32).to(torch.bfloat16), case["group"], True)
        z = y @ W.t()
        z -= z.max(dim=1, keepdim=True).values
        p = torch.exp(z)
        total = p.sum(dim=1)
        entropy.append(torch.log(total) - (p * z).sum(dim=1) / total)
        maxprob.append(1.0 / total)
    return {"argmax": None, "entropy": torch.cat(entropy), "maxprob": torch.cat(maxprob), "exit_mask": None}


def _exact_policy(case, s):
    ce, old, adv = s["ce"].to(torch.float64), s["old_ce"].to(torch.float64), s["adv"].to(torch.float64)
    use = (s["labels"] >= 0).to(torch.float64)
    n = ce.numel()
    if s["seq_start"] is None:
        share = use / max(float(use.sum()), 1.0)
    else:
        start = s["seq_start"].long()
        upto = torch.cat([use.new_zeros(1), torch.cumsum(use, 0)])
        have = upto[start[1:]] - upto[start[:-1]]
        of = torch.searchsorted(start[1:].contiguous(), torch.arange(n, device=ce.device), right=True)
        share = use / (have[of].clamp(min=1.0) * case["seqs"])
        adv = adv[of]
    ratio = torch.exp(old - ce)
    free, held = ratio * adv, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv
    cut = (held < free).to(torch.float64)
    gap = ce - s["ref_ce"].to(torch.float64)
    kl = (torch.expm1(gap) - gap) if case["kl"] > 0 else torch.zeros_like(gap)
    policy = -torch.minimum(free, held)
    dce = share * (free * (1 - cut) + case["kl"] * (torch.expm1(gap) if case["kl"] > 0 else 0.0))
    return {"loss": torch.stack([(share * (policy + case["kl"] * kl)).sum(), (share * policy).sum(), (share * kl).sum(), (share * cut).sum()]), "dce": dce}


def _exact_preference(case, s):
    use = (s["labels"] >= 0).to(torch.float64)
    worth = use * ((s["ref_ce"].to(torch.float64) if case["reference"] else 0.0) - s["ce"].to(torch.float64))
    start = s["seq_start"].tolist()
    sums = torch.stack([worth[a:b].sum() for a, b in zip(start[:-1], start[1:])]) * s["beta"]
    good, bad = sums[0::2], sums[1::2]
    margin = good - bad
    up = torch.log1p(torch.exp(-margin.abs())) + (-margin).clamp(min=0)          # -log sigmoid(margin)
    down = up + margin
    loss = (1 - s["smoothing"]) * up + s["smoothing"] * down
    slope = (1 / (1 + torch.exp(-margin)) - (1 - s["smoothing"])) * s["beta"] / case["pairs"]
    dce = torch.zeros_like(use)
    both = torch.stack([-slope, slope], dim=1).reshape(-1).tolist()
    for a, b, g in zip(start[:-1], start[1:], both):
        dce[a:b] = use[a:b] * g
    return {"loss": torch.stack([loss.mean(), (margin > 0).to(torch.float64).mean(), good.mean(), bad.mean()]), "margin": margin, "dce": dce}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "policy":
        return _exact_policy(case, s)
    if case["op"] == "preference":
        return _exact_preference(case, s)
    if case["op"] == "clip":
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(g.to(torch.float64))) ** 2 for g in s["grads"]))
        factor = min(1.0, s["max_norm"] / (norm + 1e-6))
        return {"norm": torch.tensor([norm], dtype=torch.float64, device=s["grads"][0].device), "grads": [g.to(torch.float64) * factor for g in s["grads"]]}
    if case["form"] == "pack":
        return _exact_values(s["W"], case["group"], False)
    return _exact_head(case, s)
