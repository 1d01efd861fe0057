"""The operators around the classifier's product: the scores of all labels from 8-bit integers, the check of drafted
labels against the classifier's probabilities, and dropout of the embeddings on their way into a training step.

  scores   `scores_quantized`: embeddings, quantised row by row on the way, times classifier rows kept in 8 bits
  relaid   `quantize_rows` and then `scores_quantized`: the classifier has just been trained, its 8-bit rows are laid out
           again before a batch is scored
  verify   `verify_drafts`: which of a sequence's drafted labels stand, and the label that follows them
  dropout  `dropout` on embeddings, `dropout_grad` on the gradient that a training step returns for them
Sizes are those of the workloads in `paper_2409_20156_amd.synth` and of the tests.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"

# The counter-based generator of the samplers, with a seed of its own kind for dropout ("dropout1" in ASCII).
K_ROW, K_WORD, K_DROPOUT = 0x9E3779B97F4A7C15, 0xD1B54A32D192ED03, 0x64726F706F757431
MIX1, MIX2 = 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _size(name):
    return 2 if name == "bf16" else 4


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one sequence's drafts over a small label set: the smallest call, latency is everything
        {"name": "verify_one", "kind": "verify", "dtype": "f32", "B": 1, "n": 4, "V": 4096, "draft": True, "pad": False},
        # a few sequences answered online over the labels of workload c2
        {"name": "verify_online", "kind": "verify", "dtype": "f32", "B": 8, "n": 5, "V": 131072, "draft": True, "pad": False},
        # drafts looked up rather than drawn (they have no probabilities), lists of unequal length, odd rows
        {"name": "verify_lookup_ragged", "kind": "verify", "dtype": "bf16", "B": 33, "n": 7, "V": 50021, "draft": False,
         "pad": True},
        # a full serving batch
        {"name": "verify_batch", "kind": "verify", "dtype": "bf16", "B": 256, "n": 4, "V": 131072, "draft": True, "pad": False},
        # all scores of one online query, classifier c2 kept in 8 bits
        {"name": "scores_one", "kind": "scores", "dtype": "bf16", "out": "f32", "B": 1, "L": 131072, "d": 768},
        # ... of a few queries
        {"name": "scores_online", "kind": "scores", "dtype": "bf16", "out": "f32", "B": 32, "L": 131072, "d": 768},
        # nothing a multiple of anything, single precision in and out
        {"name": "scores_ragged_f32", "kind": "scores", "dtype": "f32", "out": "f32", "B": 300, "L": 50021, "d": 300},
        # all scores of a large batch: an evaluation pass over classifier c2
        {"name": "scores_eval", "kind": "scores", "dtype": "bf16", "out": "bf16", "B": 4096, "L": 131072, "d": 768},
        # classifier c3 laid out in 8 bits after a training epoch, then a small batch scored
        {"name": "relaid_c3", "kind": "relaid", "dtype": "bf16", "out": "bf16", "B": 64, "L": 670000, "d": 768},
        # the embeddings of workload tiny: launch latency
        {"name": "dropout_tiny", "kind": "dropout", "grad": False, "dtype": "f32", "B": 32, "d": 64, "rate": 0.1},
        # the whole pool of workload c2
        {"name": "dropout_pool", "kind": "dropout", "grad": False, "dtype": "bf16", "B": 10240, "d": 768, "rate": 0.1},
        # the gradient of a pool of workload c4, rounded to the embeddings' type
        {"name": "dropout_grad", "kind": "dropout", "grad": True, "dtype": "bf16", "B": 65536, "d": 768, "rate": 0.25},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["scores", "scores", "relaid", "verify", "verify", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "dropout":
        d, B = _log(rng, 64, 8192), _log(rng, 1, 65536)
        while B * d > 5e7:
            B = int(B * 0.7)
        return {"kind": kind, "grad": rng.random() < 0.5, "dtype": dtype, "B": B, "d": d,
                "rate": rng.choice([0.05, 0.1, 0.25, 0.5])}
    if kind == "verify":
        B, n, V = _log(rng, 1, 256), rng.randint(0, 8), _log(rng, 1000, 262144)
        while B * (n + 1) * V > 1.6e8:
            B = max(1, int(B * 0.7))
        return {"kind": kind, "dtype": dtype, "B": B, "n": n, "V": V, "draft": rng.random() < 0.75, "pad": rng.random() < 0.3}
    per = 8 if dtype == "bf16" else 4                     # elements of 16 bytes, the granularity of a row
    d = max(8, _log(rng, 64, 4096) // per) * per
    d = min(d, 4096)
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


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case, "seed": seed}
    kind = case["kind"]
    if kind == "dropout":
        # embeddings, or the fp32 gradient of the loss averaged over a batch
        s["x"] = _matrix(g, case["B"], case["d"], torch.float32 if case["grad"] else _type(case["dtype"]))
        if case["grad"]:
            s["x"] /= case["B"]
        return s
    if kind == "verify":
        B, n, V, dtype = case["B"], case["n"], case["V"], _type(case["dtype"])
        logits = torch.empty((B, n + 1, V), device=DEV).normal_(0.0, 2.5, generator=g)
        if not case["draft"]:                             # looked-up labels: four in five are what the target expects as well
            s["draft"] = None
            at = torch.randint(0, V, (B, n, 1), generator=g, device=DEV)
            hit = torch.rand((B, n, 1), generator=g, device=DEV) < 0.8
            sure = logits[:, :n].logsumexp(-1, keepdim=True) + 2.0
            logits[:, :n].scatter_(2, at, torch.where(hit, sure, logits[:, :n].gather(2, at)))
            s["drafts"] = at[:, :, 0].to(torch.int32)
        s["target"] = logits.softmax(-1).to(dtype)
        if case["draft"]:
            # the draft model's logits are the target's with an error of 0.6: about three drafts in four stand
            logits = logits[:, :n] + torch.empty((B, n, V), device=DEV).normal_(0.0, 0.6, generator=g)
            s["draft"] = logits.softmax(-1).to(dtype)
            noise = torch.empty_like(logits).exponential_(generator=g)
            s["drafts"] = (logits - noise.log()).argmax(-1).to(torch.int32).reshape(B, n)          # drawn from the draft's soft-max
        if case["pad"] and n:
            have = torch.randint(0, n + 1, (B, 1), generator=g, device=DEV)
            s["drafts"][torch.arange(n, device=DEV)[None, :] >= have] = -1
        s["u"] = torch.rand((B, n + 1), generator=g, device=DEV)
        return s
    s["z"] = _matrix(g, case["B"], case["d"], _type(case["dtype"]))
    w = _matrix(g, case["L"], case["d"], _type(case["dtype"]))
    if kind == "relaid":
        s["w"] = w
    else:                                                 # 8-bit rows, padded with zeros to a multiple of 16 bytes
        m = w.float().abs().amax(1)
        q = torch.zeros((case["L"], -(-case["d"] // 16) * 16), dtype=torch.int8, device=DEV)
        q[:, :case["d"]] = torch.round(w.float() * (127.0 / m)[:, None]).to(torch.int8)
        s["q"], s["scale"] = q, m / 127.0
    return s


# ---------------------------------------------------------------------------------------------------------------
# the operators in their plain form
# ---------------------------------------------------------------------------------------------------------------
def _plain_rows(x):
    """8-bit integers (as fp32) and scale of each row; which integer is nearest is decided in 64 bits."""
    m = x.abs().amax(1, keepdim=True)
    q = torch.round(x.double() * 127.0 / m.double())
    return torch.where(m == 0, torch.zeros_like(q), q).float(), (m.double() / 127.0).float()


def _plain_scores(z, wq, ws, out):
    zq, zs = _plain_rows(z)
    return ((zq @ wq[:, :zq.shape[1]].t()).mul_(zs).mul_(ws[None, :])).to(out)


def _plain_verify(drafts, target, draft, u):
    B, n = drafts.shape
    V = target.shape[2]
    every = torch.arange(B, device=DEV)
    live = ((drafts >= 0) & (drafts < V)).cumprod(1).bool()
    at = drafts.clamp(0, V - 1).long()[:, :, None]
    p = target[:, :n].gather(2, at)[:, :, 0].double()
    q = draft.gather(2, at)[:, :, 0].double() if draft is not None else torch.ones_like(p)
    stands = (live & (u[:, :n].double() * q < p)).cumprod(1)
    a = stands.sum(1)
    fell = a < live.sum(1)
    p = target[every, a].double()
    w = p
    if n:
        b = a.clamp(max=n - 1)
        if draft is not None:
            w = p - draft[every, b].double() * fell[:, None]
        else:
            w = p.clone()
            w[every, at[every, b, 0]] *= ~fell
    w = torch.where((w > 0) & (w < math.inf), w, torch.zeros_like(w))
    p = torch.where((p > 0) & (p < math.inf), p, torch.zeros_like(p))
    w = torch.where(w.sum(1, keepdim=True) > 0, w, p)
    run_sum = w.cumsum(1)
    above = run_sum > u[:, n:].double() * run_sum[:, -1:]
    last = V - 1 - (w > 0).flip(1).to(torch.uint8).argmax(1)
    token = torch.where(above.any(1), above.to(torch.uint8).argmax(1), last)
    token = torch.where(run_sum[:, -1] > 0, token, torch.full_like(token, -1))
    out = torch.full((B, n + 1), -1, dtype=torch.int32, device=DEV)
    out[:, :n] = torch.where(stands.bool(), drafts, out[:, :n])
    out[every, a] = token.to(torch.int32)
    return out, a.to(torch.int32)


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _plain_mix(x):
    x = (x ^ ((x >> 30) & ((1 << 34) - 1))) * _signed(MIX1)
    x = (x ^ ((x >> 27) & ((1 << 37) - 1))) * _signed(MIX2)
    return x ^ ((x >> 31) & ((1 << 33) - 1))


def _plain_dropout(x, rate, seed, out):
    B, d = x.shape
    least = int(rate * 65536 + 0.5)
    row = _plain_mix((torch.arange(1, B + 1, device=DEV) * _signed(K_ROW)) ^ _signed(seed ^ K_DROPOUT))
    word = _plain_mix(row[:, None] + torch.arange(1, -(-d // 4) + 1, device=DEV)[None, :] * _signed(K_WORD))
    field = (word[:, :, None] >> torch.arange(0, 64, 16, device=DEV)) & 0xFFFF
    kept = field.reshape(B, -1)[:, :d] >= least
    return torch.where(kept, x.float() * (65536.0 / (65536 - least)), torch.zeros((), device=DEV)).to(out)


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def _own(s):
    import paper_2409_20156_amd as xc
    c = s["case"]
    kind = c["kind"]
    if kind == "dropout":
        if "out" not in s:
            s["out"] = torch.empty(s["x"].shape, dtype=_type(c["dtype"]), device=DEV)
        return (xc.dropout_grad if c["grad"] else xc.dropout)(s["x"], c["rate"], s["seed"], out=s["out"])
    if kind == "verify":
        if "out" not in s:
            s["ws"] = torch.empty(xc.verify_workspace(c["B"], c["V"]), dtype=torch.uint8, device=DEV)
            s["out"] = (torch.empty((c["B"], c["n"] + 1), dtype=torch.int32, device=DEV),
                        torch.empty(c["B"], dtype=torch.int32, device=DEV))
        return xc.verify_drafts(s["drafts"], s["target"], s["draft"], s["u"], workspace=s["ws"], out=s["out"])
    if "out" not in s:                                    # buffers that a serving program allocates once
        s["ws"] = torch.empty(xc.scores_workspace(c["B"], c["d"]), dtype=torch.uint8, device=DEV)
        s["out"] = torch.empty((c["B"], c["L"]), dtype=_type(c["out"]), device=DEV)
        if kind == "relaid":
            s["rows"] = (torch.empty((c["L"], xc.quantized_pitch(c["d"])), dtype=torch.int8, device=DEV),
                         torch.empty(c["L"], dtype=torch.float32, device=DEV))
    q, scale = xc.quantize_rows(s["w"], out=s["rows"]) if kind == "relaid" else (s["q"], s["scale"])
    return xc.scores_quantized(s["z"], q, scale, workspace=s["ws"], out=s["out"])


def run(s):
    if own:
        return _own(s)
    c = s["case"]
    if c["kind"] == "dropout":
        return _plain_dropout(s["x"], c["rate"], s["seed"], _type(c["dtype"]))
    if c["kind"] == "verify":
        return _plain_verify(s["drafts"], s["target"], s["draft"], s["u"])
    if c["kind"] == "relaid":
        wq, ws = _plain_rows(s["w"])
        return _plain_scores(s["z"], wq, ws[:, 0], _type(c["out"]))
    return _plain_scores(s["z"], s["q"].float(), s["scale"], _type(c["out"]))


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(c):
    if c["kind"] == "dropout":
        e = (4 if c["grad"] else _size(c["dtype"])) + _size(c["dtype"])
        return {"bytes": e * c["B"] * c["d"], "flops": c["B"] * c["d"]}
    if c["kind"] == "verify":
        # one row of the target per sequence, and one of the draft where a draft fell: each stands with about 0.77
        drafts = c["n"] / 2 if c["pad"] else c["n"]
        rows = 1 + (1 - 0.77 ** drafts if c["draft"] else 0)
        small = drafts * (4 + _size(c["dtype"]) * (2 if c["draft"] else 1)) + 4 * (c["n"] + 1) + 4 * (c["n"] + 2)
        return {"bytes": c["B"] * (c["V"] * _size(c["dtype"]) * rows + small), "flops": 3 * c["B"] * c["V"]}
    B, L, d = c["B"], c["L"], c["d"]
    rows = L * (d * _size(c["dtype"]) + d + 4) if c["kind"] == "relaid" else L * (d + 4)
    return {"bytes": rows + B * d * _size(c["dtype"]) + B * L * _size(c["out"]), "flops": 2 * B * L * d}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _exact_integers(x):
    """Rows of x as integers: 127 x / m to the nearest, m the largest magnitude of the row, halves to even; and m / 127."""
    x = x.to(torch.float64)
    m = torch.linalg.vector_norm(x, ord=math.inf, dim=1)
    q = (x * 127).div_(m.clamp(min=torch.finfo(torch.float64).tiny)[:, None])
    low = q.floor()
    up = q - low
    low += ((up > 0.5) | ((up == 0.5) & (torch.remainder(low, 2) == 1))).double()
    return low, m / 127


def _exact_word(x):
    with np.errstate(over="ignore"):
        x = (x ^ (x >> np.uint64(30))) * np.uint64(MIX1)
        x = (x ^ (x >> np.uint64(27))) * np.uint64(MIX2)
        return x ^ (x >> np.uint64(31))


def _exact_dropout(s, c):
    B, d = c["B"], c["d"]
    least = math.floor(65536 * c["rate"] + 0.5)
    x = s["x"].cpu().to(torch.float64).numpy()
    with np.errstate(over="ignore"):
        i = np.arange(1, B + 1, dtype=np.uint64) * np.uint64(K_ROW)
        row = _exact_word(np.uint64(s["seed"] ^ K_DROPOUT) ^ i)
        j = np.arange(d, dtype=np.uint64)
        for b in range(B):
            word = _exact_word(row[b] + (j[::4] // np.uint64(4) + np.uint64(1)) * np.uint64(K_WORD))
            field = word.astype("<u8").view("<u2")[:d]
            x[b] = np.where(field >= least, x[b] * 65536 / (65536 - least), 0.0)
    return torch.from_numpy(x)


def _exact_verify(s, c):
    B, n, V = c["B"], c["n"], c["V"]
    drafts, u = s["drafts"].cpu().tolist(), s["u"].cpu().double().numpy()
    tokens, accepted = np.full((B, n + 1), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    for b in range(B):
        a, w = 0, None
        while a < n and 0 <= drafts[b][a] < V:
            x = drafts[b][a]
            q = float(s["draft"][b, a, x]) if c["draft"] else 1.0
            if u[b, a] * q >= float(s["target"][b, a, x]):
                w = s["target"][b, a].cpu().double().numpy()
                if c["draft"]:
                    w = np.maximum(w - s["draft"][b, a].cpu().double().numpy(), 0)
                else:
                    w[x] = 0
                break
            tokens[b, a] = x
            a += 1
        if w is None or w.sum() == 0:
            w = s["target"][b, a].cpu().double().numpy()
        edge = np.cumsum(w)
        tokens[b, a] = min(int(np.searchsorted(edge, u[b, n] * edge[-1], side="right")), int(np.flatnonzero(w)[-1]))
        accepted[b] = a
    return torch.from_numpy(tokens), torch.from_numpy(accepted)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "dropout":
        return _exact_dropout(s, case)
    if case["kind"] == "verify":
        return _exact_verify(s, case)
    zq, zs = _exact_integers(s["z"])
    if case["kind"] == "relaid":
        wq, ws = _exact_integers(s["w"])
    else:
        wq, ws = s["q"][:, :case["d"]].double(), s["scale"].double()
    return (zq @ wq.t()).mul_(zs[:, None]).mul_(ws[None, :])
