"""The operators by which the classifier's scores are answered with and learnt from: the scores of all labels from 4-bit floating
point with shared scales, the log probabilities of given labels with entropy and top alternatives, their gradient, and the loss
against a teacher's top labels with its gradient.

  micro     `scores_microscaled`: embeddings, brought to 4 bits on the way, times classifier rows kept in 4 bits
  remicro   `microscale_rows` and then `scores_microscaled`: the classifier has just been trained, its 4-bit rows are laid out again
            before a batch is scored
  logprobs  `label_logprobs`: log probabilities of given labels under the soft-max of the scores, its entropy, its top labels
  policy    `label_logprobs` and then `label_logprobs_grad`: a step of training on labels that were drawn from the scores, with a
            reward for their log probabilities and one for the entropy
  distill   `distill`: the divergence from a teacher's distribution, of which the top labels are given, and its gradient
Sizes are those of the workloads in `paper_2409_20156_amd.synth` and of the tests.
"""
import math

import torch

own = False
DEV = "cuda:0"


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _size(name):
    return 2 if name == "bf16" else 4


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one query answered over a small label set, five alternatives beside the answer: the smallest call
        {"name": "logprobs_one", "kind": "logprobs", "dtype": "f32", "B": 1, "V": 4096, "n": 1, "top": 5, "temp": 1.0, "mask": 0.0,
         "pad": False},
        # a few queries answered online over the labels of workload c2, twenty alternatives, drawn at a lower temperature
        {"name": "logprobs_online", "kind": "logprobs", "dtype": "f32", "B": 8, "V": 131072, "n": 1, "top": 20, "temp": 0.7,
         "mask": 0.0, "pad": False},
        # several labels of interest per query in lists of unequal length, odd rows, half of the labels not allowed
        {"name": "logprobs_ragged", "kind": "logprobs", "dtype": "bf16", "B": 33, "V": 50021, "n": 7, "top": 3, "temp": 1.0,
         "mask": 0.5, "pad": True},
        # a teacher's pass over classifier c2: the labels and log probabilities that a student is trained on
        {"name": "logprobs_teacher", "kind": "logprobs", "dtype": "bf16", "B": 2048, "V": 131072, "n": 4, "top": 64, "temp": 1.0,
         "mask": 0.0, "pad": True},
        # a step of training on drawn labels, a small label set
        {"name": "policy_small", "kind": "policy", "dtype": "f32", "B": 32, "V": 4096, "n": 1, "temp": 1.0, "mask": 0.0, "pad": False},
        # ... a batch over classifier c2, eight labels drawn for each query
        {"name": "policy_batch", "kind": "policy", "dtype": "bf16", "B": 1024, "V": 131072, "n": 8, "temp": 1.0, "mask": 0.0,
         "pad": True},
        # a student of a small label set
        {"name": "distill_small", "kind": "distill", "dtype": "f32", "B": 32, "V": 4096, "K": 16, "temp": 1.0, "tail": False,
         "mask": 0.0, "pad": False},
        # nothing a multiple of anything, single precision, the teacher's other labels as one; labels that are not allowed
        {"name": "distill_ragged", "kind": "distill", "dtype": "f32", "B": 300, "V": 50021, "K": 33, "temp": 2.0, "tail": True,
         "mask": 0.3, "pad": True},
        # a batch over classifier c2 against the top labels of its teacher
        {"name": "distill_batch", "kind": "distill", "dtype": "bf16", "B": 1024, "V": 131072, "K": 64, "temp": 1.0, "tail": True,
         "mask": 0.0, "pad": False},
        # all scores of one online query, classifier c2 kept in 4 bits
        {"name": "micro_one", "kind": "micro", "dtype": "bf16", "out": "f32", "B": 1, "L": 131072, "d": 768},
        # all scores of a large batch: an evaluation pass over classifier c2
        {"name": "micro_eval", "kind": "micro", "dtype": "bf16", "out": "bf16", "B": 4096, "L": 131072, "d": 768},
        # classifier c3 laid out in 4 bits after a training epoch, then a small batch scored
        {"name": "remicro_c3", "kind": "remicro", "dtype": "bf16", "out": "bf16", "B": 64, "L": 670000, "d": 768},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprobs", "logprobs", "policy", "distill", "distill", "micro", "micro", "remicro"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("logprobs", "policy", "distill"):
        B, V = _log(rng, 1, 4096), _log(rng, 1000, 262144)
        while B * V > (2.0e8 if kind == "logprobs" else 1.0e8):
            B = max(1, int(B * 0.7))
        c = {"kind": kind, "dtype": dtype, "B": B, "V": V, "temp": rng.choice([0.7, 1.0, 1.0, 2.0]),
             "mask": rng.choice([0.0, 0.0, 0.3, 0.6]), "pad": rng.random() < 0.5}
        if kind == "distill":
            c.update(K=_log(rng, 1, 128), tail=rng.random() < 0.5)
        else:
            c.update(n=_log(rng, 1, 16))
        if kind == "logprobs":
            c.update(top=rng.choice([0, 1, 5, 10, 20, 64, 128]))
        return c
    per = 8 if dtype == "bf16" else 4                     # elements of 16 bytes, the granularity of a row
    d = min(4096, max(8, _log(rng, 64, 4096) // per * per))
    if rng.random() < 0.3:
        d = rng.choice([64, 128, 192, 256, 384, 512, 768])
    B, L = _log(rng, 1, 4096), _log(rng, 1000, 1300000)
    while B * L * d > 4e11 or B * L > 5e8 or L * d > 5e8:
        if B > 64 and rng.random() < 0.5:
            B = int(B * 0.7)
        else:
            L = int(L * 0.7)
    return {"kind": kind, "dtype": dtype, "out": rng.choice(["bf16", "f32"]), "B": B, "L": L, "d": d}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _matrix(g, n, d, dtype):
    """Rows of entries N(0, 1/d), their lengths spread by about a third."""
    x = torch.empty((n, d), dtype=torch.float32, device=DEV).normal_(0.0, d ** -0.5, generator=g)
    x *= torch.empty((n, 1), device=DEV).normal_(0.0, 0.3, generator=g).exp_()
    return x.to(dtype)


def _some(g, labels, pad):
    """Lists of labels, ended early by -1 where they are to be of unequal length."""
    B, n = labels.shape
    labels = labels.to(torch.int32)
    if pad:
        have = torch.randint(0, n + 1, (B, 1), generator=g, device=DEV)
        labels[torch.arange(n, device=DEV)[None, :] >= have] = -1
    return labels


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind in ("micro", "remicro"):
        s["z"] = _matrix(g, case["B"], case["d"], _type(case["dtype"]))
        w = _matrix(g, case["L"], case["d"], _type(case["dtype"]))
        if kind == "remicro":
            s["w"] = w
        else:                                             # 4-bit rows, laid out once
            s["q"], s["scale"] = _packed(*_plain_micro(w))
        return s
    B, V, T = case["B"], case["V"], case["temp"]
    x = torch.empty((B, V), device=DEV).normal_(0.0, 2.5, generator=g)
    if case["mask"]:
        x[torch.rand((B, V), generator=g, device=DEV) < case["mask"]] = -math.inf
    s["x"] = x.to(_type(case["dtype"]))
    if kind == "distill":
        # the teacher's logits are the student's with an error of 1; a row in eight is left out of the batch by its weight
        x = x + torch.empty((B, V), device=DEV).normal_(0.0, 1.0, generator=g)
        t = (x / T).log_softmax(-1)
        top = t.topk(min(case["K"], V), dim=-1)
        s["labels"] = _some(g, top.indices, case["pad"])
        s["teacher"] = top.values.contiguous()
        s["weight"] = torch.full((B,), 1.0 / B, device=DEV)
        s["weight"][torch.rand((B,), generator=g, device=DEV) < 0.125] = 0.0
        return s
    n = case["n"]
    drawn = [(x / T - torch.empty_like(x).exponential_(generator=g).log()).argmax(-1) for _ in range(n)]      # from the soft-max
    s["labels"] = _some(g, torch.stack(drawn, 1), case["pad"])
    if kind == "policy":
        s["dlogp"] = torch.empty((B, n), device=DEV).normal_(0.0, 1.0 / (B * n), generator=g)
        s["dentropy"] = torch.full((B,), -0.01 / B, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------------------
# the operators in their plain form
# ---------------------------------------------------------------------------------------------------------------
def _plain_micro(x):
    """Rows in blocks of 32: the elements' values on the 4-bit grid [N, blocks, 32], and the blocks' binary exponents [N, blocks]."""
    N, d = x.shape
    pitch = -(-d // 128) * 128
    v = torch.zeros((N, pitch), device=DEV)
    v[:, :d] = x
    v = v.view(N, pitch // 32, 32)
    e = torch.frexp(v.abs().amax(2))[1] - 3               # floor(log2 of the largest) - 2, the exponent of 4
    e = torch.where((v != 0).any(2), e, torch.full_like(e, -127)).clamp(min=-127)
    a = torch.ldexp(v.double(), -e[:, :, None]).abs()
    g = torch.zeros_like(v)
    for at, step in ((0.25, 0.5), (0.75, 0.5), (1.25, 0.5), (1.75, 0.5), (2.5, 1.0), (3.5, 1.0), (5.0, 2.0)):
        g += step * ((a >= at) if at in (0.75, 1.75, 3.5) else (a > at))               # halves to the even code
    return torch.where(v < 0, -g, g), e


def _packed(v, e):
    """Values as codes (sign, two bits of exponent, one of mantissa), two to a byte, the lower first; exponents as bytes."""
    N = v.shape[0]
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    code = torch.bucketize(v.abs(), grid).to(torch.uint8)
    code = torch.where(torch.signbit(v), code + 8, code).view(N, -1)
    return code[:, ::2] | (code[:, 1::2] << 4), (e + 127).to(torch.uint8)


def _unpacked(q, scale):
    """Rows of fp32 from what `_packed` gives."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    grid = torch.cat([grid, -grid])
    v = torch.stack([grid[(q & 15).int()], grid[(q >> 4).int()]], 2).view(q.shape[0], -1, 32)
    return torch.ldexp(v, scale.int()[:, :, None] - 127).view(q.shape[0], -1)


def _values(v, e):
    return torch.ldexp(v, e[:, :, None]).view(v.shape[0], -1)


def _plain_stats(x, T):
    """Largest score m, (x - m) / T, its exponential, and the sum of these; a row without labels sums to 0."""
    m = x.amax(1, keepdim=True)
    d = (x - torch.where(m == -math.inf, torch.zeros_like(m), m)) / T
    e = d.exp()
    return m, d, e, e.sum(1, keepdim=True)


def _plain_logprobs(x, labels, T, top):
    x = x.float()
    B, V = x.shape
    m, d, e, s = _plain_stats(x, T)
    norm = s.log()
    there = (labels >= 0) & (labels < V)
    logp = d.gather(1, labels.clamp(0, V - 1).long()) - norm
    logp = torch.where(there, logp, torch.zeros_like(logp))
    entropy = norm[:, 0] - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1) / s[:, 0]
    out = {"logp": logp, "entropy": entropy, "norm": torch.cat([m, norm], 1)}
    if top:
        # larger score first, then the lower label: both in one whole number
        i = (x + 0.0).view(torch.int32).long()
        key = torch.where(i >= 0, i, i ^ 0x7FFFFFFF) * (1 << 32) + ((1 << 32) - 1 - torch.arange(V, device=DEV)[None, :])
        at = ((1 << 32) - 1 - (key.topk(min(top, V), 1).values & 0xFFFFFFFF))
        value = d.gather(1, at) - norm
        none = value == -math.inf
        out["top"] = torch.where(none, torch.full_like(at, -1), at).to(torch.int32)
        out["top_logp"] = value
    return out


def _plain_policy(x, labels, dlogp, dentropy, T, out):
    r = _plain_logprobs(x, labels, T, 0)
    V = x.shape[1]
    there = (labels >= 0) & (labels < V)
    g = torch.where(there, dlogp, torch.zeros_like(dlogp))
    logp = (x.float() - r["norm"][:, :1]) / T - r["norm"][:, 1:]
    p = logp.exp()
    inner = g.sum(1, keepdim=True) + dentropy[:, None] * (logp + r["entropy"][:, None])
    dx = torch.where(p > 0, -p * inner, torch.zeros_like(p))
    dx.scatter_add_(1, labels.clamp(0, V - 1).long(), g)
    return {"logp": r["logp"], "entropy": r["entropy"], "dx": (dx / T).to(out)}


def _plain_distill(x, labels, teacher, weight, T, tail, out):
    x = x.float()
    B, V = x.shape
    there = (labels >= 0) & (labels < V)
    at = labels.clamp(0, V - 1).long()
    t = torch.where(there, teacher.double(), torch.full((), -math.inf, dtype=torch.float64, device=DEV))
    if not tail:
        m = t.amax(1, keepdim=True)
        t = t - torch.where(m == -math.inf, torch.zeros_like(m), m)
        t = t - t.exp().sum(1, keepdim=True).log()
    q = torch.where(there, t.exp(), torch.zeros_like(t))
    m, d, e, s = _plain_stats(x, T)
    s = s.double()
    if tail:
        # the labels that are not listed, as one: the teacher's probability of them, the student's, and each one's share.  The sum over
        # all labels is the listed ones' and the others', so that what both err by leaves their ratio alone
        listed_ = torch.zeros((B, V), dtype=torch.bool, device=DEV)
        listed_.scatter_(1, torch.where(there, at, at[:, :1]), there | there[:, :1])
        mr, _, er, sr = _plain_stats(torch.where(listed_, torch.full_like(x, -math.inf), x), T)
        others = torch.where(sr > 0, ((mr - m).double() / T).exp() * sr.double(), torch.zeros_like(s))
        s = others + torch.where(listed_, e, torch.zeros_like(e)).sum(1, keepdim=True, dtype=torch.float64)
    logs = s.log()
    safe = torch.where(m == -math.inf, torch.zeros_like(m), m).double()
    logp = (x.gather(1, at).double() - safe) / T - logs
    loss = torch.where(q > 0, q * (t - logp), torch.zeros_like(q)).sum(1)
    p = (d - logs.float()).exp()
    if tail:
        rest = (1.0 - q.sum(1, keepdim=True)).clamp(min=0)
        rest = torch.where(sr > 0, rest, torch.zeros_like(rest))
        logr = sr.double().log() + torch.where(mr == -math.inf, mr, mr - m).double() / T - logs
        loss = loss + torch.where(rest > 0, rest * (rest.log() - logr), torch.zeros_like(rest))[:, 0]
        mass = q.sum(1, keepdim=True) + rest
        share = er / torch.where(sr > 0, sr, torch.ones_like(sr))
        p = torch.where(listed_, p * mass.float(), (mass * logr.exp() - rest).float() * share)
    p.scatter_add_(1, at, -q.float())
    live = (weight != 0) & there.any(1)
    loss = torch.where(live, weight * T * T * loss, torch.zeros_like(loss))
    dx = torch.where(live[:, None], p * (weight * T)[:, None], torch.zeros_like(p))
    return {"loss": loss.float(), "dx": dx.to(out)}


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2409_20156_amd as xc
    c = s["case"]
    kind = c["kind"]
    code = xc.XC_BF16 if c["dtype"] == "bf16" else xc.XC_F32
    first = "out" not in s                                # buffers that a program allocates once
    if kind in ("micro", "remicro"):
        if first:
            s["ws"] = torch.empty(xc.scores_microscaled_workspace(c["B"], c["d"]), dtype=torch.uint8, device=DEV)
            s["out"] = torch.empty((c["B"], c["L"]), dtype=_type(c["out"]), device=DEV)
            if kind == "remicro":
                pitch = xc.microscaled_pitch(c["d"])
                s["rows"] = (torch.empty((c["L"], pitch // 2), dtype=torch.uint8, device=DEV),
                             torch.empty((c["L"], pitch // 32), dtype=torch.uint8, device=DEV))
        q, scale = xc.microscale_rows(s["w"], out=s["rows"]) if kind == "remicro" else (s["q"], s["scale"])
        return xc.scores_microscaled(s["z"], q, scale, workspace=s["ws"], out=s["out"])
    B, V = c["B"], c["V"]
    if kind == "distill":
        if first:
            s["ws"] = torch.empty(xc.distill_workspace(B, V, code), dtype=torch.uint8, device=DEV)
            s["out"] = (torch.empty(B, device=DEV), torch.empty((B, V), dtype=_type(c["dtype"]), device=DEV))
        loss, dx = xc.distill(s["x"], s["labels"], s["teacher"], temperature=c["temp"], tail=c["tail"], weight=s["weight"],
                              workspace=s["ws"], out=s["out"])
        return {"loss": loss, "dx": dx}
    top = min(c.get("top", 0), V)
    if first:
        n = c["n"]
        s["ws"] = torch.empty(xc.label_logprobs_workspace(B, V, top, code), dtype=torch.uint8, device=DEV)
        s["out"] = {"logp": torch.empty((B, n), device=DEV), "entropy": torch.empty(B, device=DEV), "norm": torch.empty((B, 2), device=DEV)}
        if top:
            s["out"].update(top=torch.empty((B, top), dtype=torch.int32, device=DEV), top_logp=torch.empty((B, top), device=DEV))
        if kind == "policy":
            s["dx"] = torch.empty((B, V), dtype=_type(c["dtype"]), device=DEV)
    r = xc.label_logprobs(s["x"], s["labels"], top=top, temperature=c["temp"], workspace=s["ws"], out=s["out"])
    if kind == "logprobs":
        return r
    dx = xc.label_logprobs_grad(s["x"], s["labels"], s["dlogp"], r["norm"], temperature=c["temp"], entropy=r["entropy"],
                                dentropy=s["dentropy"], out=s["dx"])
    return {"logp": r["logp"], "entropy": r["entropy"], "dx": dx}


def run(s):
    if own:
        return _own(s)
    c = s["case"]
    if c["kind"] == "micro":
        z = _values(*_plain_micro(s["z"]))
        return (z @ _unpacked(s["q"], s["scale"]).t()).to(_type(c["out"]))
    if c["kind"] == "remicro":
        z, w = _values(*_plain_micro(s["z"])), _values(*_plain_micro(s["w"]))
        return (z @ w.t()).to(_type(c["out"]))
    if c["kind"] == "distill":
        return _plain_distill(s["x"], s["labels"], s["teacher"], s["weight"], c["temp"], c["tail"], _type(c["dtype"]))
    if c["kind"] == "policy":
        return _plain_policy(s["x"], s["labels"], s["dlogp"], s["dentropy"], c["temp"], _type(c["dtype"]))
    return _plain_logprobs(s["x"], s["labels"], c["temp"], c["top"])


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(c):
    B = c["B"]
    if c["kind"] in ("micro", "remicro"):
        L, d = c["L"], c["d"]
        rows = L * (d / 2 + d / 32) + (L * d * _size(c["dtype"]) if c["kind"] == "remicro" else 0)
        return {"bytes": rows + B * d * _size(c["dtype"]) + B * L * _size(c["out"]), "flops": 2 * B * L * d}
    V, e = c["V"], _size(c["dtype"])
    if c["kind"] == "distill":
        return {"bytes": B * (2 * V * e + 8 * c["K"] + 8), "flops": 8 * B * V}
    if c["kind"] == "policy":
        return {"bytes": B * (2 * V * e + 12 * c["n"] + 8), "flops": 10 * B * V}
    return {"bytes": B * (V * e + 8 * c["n"] + 8 * c["top"] + 12), "flops": 5 * B * V}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_micro(x):
    """Blocks of 32 of a row: x / 2^e to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (halves to the even neighbour, beyond 6 is 6), times 2^e,
    with e = floor(log2(largest magnitude)) - 2."""
    x = x.double()
    N, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % 128)).view(N, -1, 32)
    big = torch.linalg.vector_norm(x, ord=math.inf, dim=2, keepdim=True)
    unit = torch.exp2((torch.floor(torch.log2(big.clamp(min=2.0 ** -125))) - 2).clamp(min=-127))
    y = x / unit
    gap = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return ((torch.round(y / gap) * gap).clamp(-6, 6) * unit).view(N, -1)


def exact(case, seed):
    s, T = prepare(case, seed), case.get("temp")
    if case["kind"] in ("micro", "remicro"):
        if case["kind"] == "remicro":
            w = _exact_micro(s["w"])
        else:
            low, high = (s["q"] % 16).long(), (s["q"] // 16).long()
            code = torch.stack([low, high], 2).view(case["L"], -1, 32)
            k = code % 8
            v = torch.where(k < 2, 0.5 * k, (1 + 0.5 * (k % 2)) * torch.exp2((k // 2 - 1).double())) * torch.where(code < 8, 1.0, -1.0)
            w = (v * torch.exp2(s["scale"].double() - 127)[:, :, None]).view(case["L"], -1)
        return _exact_micro(s["z"]) @ w.t()
    x = s["x"].double() / T
    B, V = x.shape
    labels = [[v for v in row if 0 <= v < V] for row in s["labels"].tolist()]
    lse = torch.logsumexp(x, 1)
    if case["kind"] == "distill":
        loss, dx = torch.zeros(B, dtype=torch.float64), torch.zeros_like(x)
        weight = s["weight"].tolist()
        for b in range(B):
            if not labels[b] or weight[b] == 0:
                continue
            at = torch.tensor(labels[b], device=DEV)
            t = s["teacher"][b, :len(labels[b])].double()
            q = t.exp() if case["tail"] else t.softmax(0)
            target = torch.zeros(V, dtype=torch.float64, device=DEV)
            target[at] = q
            logp = x[b] - lse[b]
            p = logp.exp()
            other = torch.ones(V, dtype=torch.bool, device=DEV)
            other[at] = False
            value = (q * (q.log() - logp[at])).sum()
            if case["tail"]:
                rest = max(0.0, float(1 - q.sum()))
                have = float(torch.logsumexp(logp[other], 0)) if len(labels[b]) < V else -math.inf
                if rest > 0 and have > -math.inf:
                    value = value + rest * (math.log(rest) - have)
                    target[other] = rest * (logp[other] - have).exp()
            loss[b] = value * weight[b] * T * T
            dx[b] = (p * target.sum() - target) * weight[b] * T
        return {"loss": loss, "dx": dx}
    logp = x - lse[:, None]
    p = logp.exp()
    entropy = -(p * logp.clamp(min=-1e300)).sum(1)
    given = s["labels"].long()
    there = (given >= 0) & (given < V)
    value = torch.where(there, logp.gather(1, given.clamp(min=0)), 0.0)
    if case["kind"] == "policy":
        dx = -p * (entropy[:, None] + logp.clamp(min=-1e300)) * s["dentropy"].double()[:, None]
        g = torch.where(there, s["dlogp"].double(), 0.0)
        dx -= p * g.sum(1, keepdim=True)
        dx.scatter_add_(1, given.clamp(min=0), g)
        return {"logp": value, "entropy": entropy, "dx": dx / T}
    big = x.amax(1)
    out = {"logp": value, "entropy": entropy, "norm": torch.stack([big * T, lse - big], 1)}
    if case["top"]:
        best, at = logp.sort(dim=1, descending=True, stable=True)
        k = min(case["top"], V)
        out["top"] = torch.where(best[:, :k] > -math.inf, at[:, :k], -1).to(torch.int32)
        out["top_logp"] = best[:, :k]
    return out
