"""What the sequence-model operators of the forecasting side are measured on.

Two operators, in the forms in which a forecaster of job profiles calls them:

* the selective state space scan with its short causal convolution: over the packed histories of many jobs ("prompt")
  and over one new step of each job ("step"), state and convolution history kept per job in slots;
* the statistics of token rows ("stats"): log probability of given tokens, entropy and the most likely alternatives.

``run`` computes them with elementary torch operations in 32 bits (``own = False``) or through the package's public
calls (``own = True``); ``exact`` computes them in 64 bits from the definition.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
PLAIN_VALUES = 1 << 28      # values of one [tokens, channels, state] array that the plain form holds at a time


# ---------------------------------------------------------------------------------------------------- cases

def _ssm(name, form, jobs, short, long, channels, state, groups, width, dtype, gate, resume):
    return {"name": name, "op": "ssm", "form": form, "jobs": jobs, "short": short, "long": long, "channels": channels,
            "state": state, "groups": groups, "width": width, "dtype": dtype, "gate": gate, "resume": resume}


def _stats(name, rows, vocab, top, dtype, scale, masked, pad):
    return {"name": name, "op": "stats", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "scale": scale,
            "masked": masked, "pad": pad}


def listed():
    return [
        # three jobs just submitted with a few dozen observed steps each: an interactive call, latency counts
        _ssm("prompt_few", "prompt", 3, 16, 48, 512, 16, 1, 4, "bf16", True, False),
        # the tiny round's job set, 64 jobs of 256 steps, through one layer of ordinary width
        _ssm("prompt_64x256", "prompt", 64, 256, 256, 1024, 16, 1, 4, "bf16", True, False),
        # heavy-tailed histories continued from kept states, odd widths, two groups, no gate
        _ssm("prompt_ragged", "prompt", 150, 16, 4096, 750, 12, 2, 3, "f16", False, True),
        # one job of the longest profile, 65 536 steps: few rows, a long axis
        _ssm("prompt_long", "prompt", 1, 65536, 65536, 1024, 16, 1, 4, "bf16", True, False),
        # a load of 64 jobs of 1024 steps through a wide layer: the largest
        _ssm("prompt_64x1024", "prompt", 64, 1024, 1024, 2048, 16, 1, 4, "bf16", True, False),
        # 32-bit activations with a larger state
        _ssm("prompt_f32", "prompt", 24, 100, 1000, 512, 64, 1, 4, "f32", True, True),
        # one job has advanced by a step: the smallest call
        _ssm("step_1", "step", 1, 1, 1, 1024, 16, 1, 4, "bf16", True, True),
        # the winners of a round of 512 gaps advance
        _ssm("step_512", "step", 512, 1, 1, 1024, 16, 1, 4, "bf16", True, True),
        # every job of the medium configuration, 4096 of them, advances
        _ssm("step_4096", "step", 4096, 1, 1, 2048, 16, 1, 4, "bf16", True, True),
        # one row of a large vocabulary: the answer to a single token
        _stats("stats_1", 1, 131072, 8, "bf16", 1.0, 0.0, 0),
        # memory bins of every job of the medium configuration, 16 steps ahead
        _stats("stats_bins", 65536, 1024, 16, "bf16", 1.0, 0.0, 0),
        # a padded, masked vocabulary of odd size at a temperature
        _stats("stats_odd", 1777, 50001, 20, "f16", 0.7, 0.3, 15),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "step", "stats", "stats"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "stats":
        vocab = _log_int(rng, 200, 131072)
        rows = _log_int(rng, 1, max(1, min(65536, (1 << 26) // vocab)))
        return {"op": "stats", "rows": rows, "vocab": vocab, "top": rng.randint(0, 24), "dtype": dtype,
                "scale": rng.choice([1.0, rng.uniform(0.4, 2.0)]), "masked": rng.choice([0.0, rng.uniform(0.05, 0.9)]),
                "pad": rng.choice([0, rng.randint(1, 40)])}
    groups = rng.choice([1, 1, 2, 4])
    channels = max(1, _log_int(rng, 64, 2048) // groups) * groups
    state = rng.choice([16, 16, 8, 32, 64, rng.randint(3, 40)])
    width = rng.choice([4, 4, 3, 2])
    case = {"op": "ssm", "form": kind, "channels": channels, "state": state, "groups": groups, "width": width,
            "dtype": dtype, "gate": rng.random() < 0.75, "resume": kind == "step" or rng.random() < 0.4}
    if kind == "step":
        most = (1 << 27) // (channels * state)
        return dict(case, jobs=_log_int(rng, 1, max(1, min(8192, most))), short=1, long=1)
    most = max(64, (1 << 30) // (channels * state))            # tokens in all
    jobs = _log_int(rng, 1, 256)
    long = _log_int(rng, 8, max(16, min(16384, most // jobs)))
    return dict(case, jobs=jobs, short=rng.randint(1, long), long=long)


def _lengths(case):
    """History lengths of the jobs: log-spaced from short to long in an order fixed by the case, some of them odd."""
    n, lo, hi = case["jobs"], case["short"], case["long"]
    if lo == hi or n == 1:
        return [hi] * n
    got = [int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    return [got[(i * 7919) % n] for i in range(n)] if n % 7919 else got


# ---------------------------------------------------------------------------------------------------- inputs

def _layer_weights(case, g):
    d, n, w, rows = case["channels"], case["state"], case["width"], case["channels"] + 2 * case["groups"] * case["state"]
    f = dict(device="cuda", dtype=torch.float32, generator=g)
    step = torch.exp(torch.rand(d, **f) * math.log(100.0) + math.log(1e-3))      # time steps of 0.001 .. 0.1
    return {"A": -(torch.arange(1, n + 1, device="cuda", dtype=torch.float32) * (0.7 + 0.6 * torch.rand(d, n, **f))).contiguous(),
            "skip": 1.0 + 0.1 * torch.randn(d, **f), "dt_bias": step + torch.log(-torch.expm1(-step)),
            "conv_w": (torch.rand(rows, w, **f) - 0.5) * (2.0 / math.sqrt(w)), "conv_b": 0.1 * torch.randn(rows, **f)}


_context = []


def _ctx():
    """The program's one library context, on the default stream."""
    if not _context:
        from paper_2509_19086_b200 import binding
        _context.append(binding.Sja())
    return _context[0]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]
    if case["op"] == "stats":
        rows, vocab = case["rows"], case["vocab"]
        wide = torch.empty(rows, vocab + case["pad"], device="cuda", dtype=t)
        logits = wide[:, :vocab]
        for a in range(0, rows, 4096):
            part = torch.randn(min(4096, rows - a), vocab, device="cuda", generator=g) * 2.5
            if case["masked"]:
                part[torch.rand(part.shape, device="cuda", generator=g) < case["masked"]] = -math.inf
            logits[a:a + 4096] = part
        tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        if case["masked"] and rows > 8:
            tokens[3], logits[5] = -1, -math.inf       # a position that is not scored; a row whose mask leaves nothing
        state = {"case": case, "logits": logits, "tokens": tokens}
        if own:
            state["ctx"] = _ctx()
        return state
    lens = _lengths(case)
    jobs, total = len(lens), sum(lens)
    d, n, w, rows = case["channels"], case["state"], case["width"], case["channels"] + 2 * case["groups"] * case["state"]
    # row, time step and gate are slices of one product's output, as a projection of all of them leaves them
    wide = torch.randn(total, rows + d + (d if case["gate"] else 0), device="cuda", generator=g).to(t)
    state = {"case": case, "lens": lens, "wide": wide, "xbc": wide[:, :rows], "dt": wide[:, rows:rows + d],
             "z": wide[:, rows + d:] if case["gate"] else None, **_layer_weights(case, g)}
    off = torch.zeros(jobs + 1, dtype=torch.int64)
    off[1:] = torch.tensor(lens).cumsum(0)
    state["off"] = off.cuda()
    state["slots"] = torch.randperm(jobs, device="cuda", generator=g).to(torch.int32)
    state["state"] = 0.3 * torch.randn(jobs, d, n, device="cuda", generator=g)
    state["history"] = torch.randn(jobs, w - 1, rows, device="cuda", generator=g).to(t)
    if own:
        state["layer"] = _ctx().ssm_layer(state["A"], conv_w=state["conv_w"], conv_b=state["conv_b"], skip=state["skip"],
                                          dt_bias=state["dt_bias"], n_groups=case["groups"])
    return state


# ---------------------------------------------------------------------------------------------------- one pass

def run(state):
    case = state["case"]
    if case["op"] == "stats":
        if own:
            return state["ctx"].token_stats(state["logits"], state["tokens"], top=case["top"], scale=case["scale"])
        return _plain_stats(state["logits"], state["tokens"], case["top"], case["scale"])
    if own:
        if case["form"] == "step":
            y = state["layer"].step(state["xbc"], state["dt"], state["state"], history=state["history"], z=state["z"], slots=state["slots"])
        else:
            y = state["layer"].prompt(state["xbc"], state["dt"], state["off"], state=state["state"], history=state["history"],
                                      z=state["z"], slots=state["slots"], resume=case["resume"])
    else:
        y = _plain_ssm(state)
    return {"y": y, "state": state["state"], "history": state["history"]}


def _plain_stats(logits, tokens, top, scale):
    x = logits.float()
    scaled = x * scale
    most = scaled.max(dim=1, keepdim=True).values
    most = torch.where(most == -math.inf, torch.zeros_like(most), most)
    e = torch.exp(scaled - most)
    total = e.sum(dim=1, keepdim=True)
    lse = most + torch.log(total)
    weighted = torch.where(e > 0, e * (scaled - most), torch.zeros_like(e)).sum(dim=1, keepdim=True)
    entropy = torch.where(total > 0, torch.log(total) - weighted / total, torch.zeros_like(total))
    at = scaled.gather(1, tokens.clamp(min=0)[:, None])
    logp = torch.where(at == -math.inf, at, at - lse)[:, 0]
    # distinct whole keys: larger logit first, then the lower index
    bits = (x + 0.0).view(torch.int32).to(torch.int64)
    order = torch.where(bits >= 0, bits, -2147483648 - bits) * 4294967296 + (4294967295 - torch.arange(x.shape[1], device=x.device))
    ids = torch.topk(order, top, dim=1).indices
    best = scaled.gather(1, ids)
    return {"logp": torch.where(tokens < 0, torch.zeros_like(logp), logp), "entropy": entropy[:, 0],
            "top_logp": torch.where(best == -math.inf, best, best - lse), "top_ids": ids.to(torch.int32)}


def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _plain_ssm(s):
    case, slots = s["case"], s["slots"].long()
    d, n, g, w = case["channels"], case["state"], case["groups"], case["width"]
    total, off = s["xbc"].shape[0], s["off"]
    job = torch.searchsorted(off, torch.arange(total, device="cuda"), right=True) - 1
    pos = torch.arange(total, device="cuda") - off[job]
    first, row = off[:-1], s["xbc"].float()
    past = s["history"].float()[slots] if case["resume"] else torch.zeros(s["history"].shape, device="cuda")
    u = s["conv_b"].expand_as(row)
    for k in range(w):
        back = w - 1 - k
        inside = (pos >= back)[:, None]
        old = past[job, (pos - back + w - 1).clamp(max=w - 2)] if back else row
        u = u + s["conv_w"][:, k] * torch.where(inside, torch.roll(row, back, 0), old)
    u = _silu(u)
    x, B, C = u[:, :d], u[:, d:d + g * n].view(total, g, n), u[:, d + g * n:].view(total, g, n)
    raw = s["dt"].float() + s["dt_bias"]
    dt = torch.clamp(raw, min=0.0) + torch.log1p(torch.exp(-raw.abs()))
    y = torch.empty(total, d, device="cuda")
    size = max(1, min(d // g, PLAIN_VALUES // (total * n)))
    for c in range(0, d, d // g):
        for a in range(c, c + d // g, size):
            b = min(a + size, c + d // g)
            h = (dt[:, a:b] * x[:, a:b])[:, :, None] * B[:, c * g // d][:, None, :]
            decay = torch.exp(dt[:, a:b, None] * s["A"][a:b])
            if case["resume"]:
                h[first] += decay[first] * s["state"][slots, a:b]
            decay[first] = 0.0
            reach = 1
            while reach < case["long"]:                # recurrence by doubling; the zero decay at a first step cuts it
                h[reach:] += decay[reach:] * h[:-reach]
                decay[reach:] *= decay[:-reach].clone()
                reach *= 2
            y[:, a:b] = (h * C[:, c * g // d][:, None, :]).sum(dim=2) + s["skip"][a:b] * x[:, a:b]
            s["state"][slots, a:b] = h[off[1:] - 1]
    if s["z"] is not None:
        y = y * _silu(s["z"].float())
    tail = off[1:, None] - (w - 1) + torch.arange(w - 1, device="cuda")
    kept = past.gather(1, (tail - first[:, None] + w - 1).clamp(0, w - 2)[:, :, None].expand_as(past))
    s["history"][slots] = torch.where((tail >= first[:, None])[:, :, None], row[tail.clamp(min=0)], kept).to(s["history"].dtype)
    return y.to(s["xbc"].dtype)


# ---------------------------------------------------------------------------------------------------- what it takes

def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "stats":
        r, v = case["rows"], case["vocab"]
        return {"bytes": r * v * e + r * (8 + 8 + 8 * case["top"]), "flops": 6 * r * v}
    lens = _lengths(case)
    s, total, d, n, w = len(lens), sum(lens), case["channels"], case["state"], case["width"]
    rows = d + 2 * case["groups"] * n
    kept = s * (d * n * 4 + (w - 1) * rows * e) * (2 if case["resume"] else 1)
    weights = 4 * (d * n + 2 * d + rows * (w + 1))
    return {"bytes": total * e * (rows + 2 * d + (d if case["gate"] else 0)) + kept + weights + 8 * (s + 1) + 4 * s,
            "flops": total * (7 * d * n + rows * (2 * w + 4) + 12 * d)}


# ---------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "stats":
        return _exact_stats(s)
    return _exact_ssm(s)


def _exact_stats(s):
    case = s["case"]
    logp, entropy, best, ids = [], [], [], []
    for a in range(0, case["rows"], 512):
        x = s["logits"][a:a + 512].double()
        l = torch.log_softmax(x * case["scale"], dim=1)
        empty = torch.isinf(x).all(dim=1)
        l[empty] = -math.inf
        p = torch.exp(l)
        entropy.append(-(p * l.clamp(min=-1e300)).sum(dim=1))
        t = s["tokens"][a:a + 512]
        picked = l[torch.arange(t.numel(), device="cuda"), t.clamp(min=0)]
        logp.append(picked.masked_fill(t < 0, 0.0))
        at = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
        ids.append(at.to(torch.int32))
        best.append(l.gather(1, at))
    return {"logp": torch.cat(logp), "entropy": torch.cat(entropy), "top_logp": torch.cat(best), "top_ids": torch.cat(ids)}


def _exact_ssm(s):
    """The recurrence step by step, all jobs at once, the longest first so that the running ones are a prefix."""
    case, lens = s["case"], s["lens"]
    if max(lens) > 70000 or sum(lens) * case["channels"] * case["state"] > 1 << 32:
        return None
    d, n, g, w = case["channels"], case["state"], case["groups"], case["width"]
    order = sorted(range(len(lens)), key=lambda j: -lens[j])
    begin = [0]
    for v in lens:
        begin.append(begin[-1] + v)
    begin = torch.tensor([begin[j] for j in order], device="cuda")
    slots = s["slots"].long()[torch.tensor(order, device="cuda")]
    h, window = s["state"].double()[slots], s["history"].double()[slots]
    if not case["resume"]:
        h, window = torch.zeros_like(h), torch.zeros_like(window)
    y = torch.empty(sum(lens), d, device="cuda", dtype=torch.float64)
    A, cw, cb, skip, bias = (s[k].double() for k in ("A", "conv_w", "conv_b", "skip", "dt_bias"))
    live = len(lens)
    for t in range(max(lens)):
        while lens[order[live - 1]] <= t:
            live -= 1
        at = begin[:live] + t
        full = torch.cat([window[:live], s["xbc"][at].double()[:, None]], dim=1)
        window[:live] = full[:, 1:]
        u = torch.nn.functional.silu((full * cw.t()).sum(dim=1) + cb)
        x = u[:, :d]
        B = u[:, d:d + g * n].reshape(live, g, 1, n).expand(live, g, d // g, n).reshape(live, d, n)
        C = u[:, d + g * n:].reshape(live, g, 1, n).expand(live, g, d // g, n).reshape(live, d, n)
        dt = torch.nn.functional.softplus(s["dt"][at].double() + bias, threshold=50.0)
        h[:live] = torch.exp(dt[:, :, None] * A) * h[:live] + (dt * x)[:, :, None] * B
        o = (h[:live] * C).sum(dim=2) + skip * x
        y[at] = o * torch.nn.functional.silu(s["z"][at].double()) if s["z"] is not None else o
    state, history = s["state"].double(), s["history"].double()
    state[slots], history[slots] = h, window
    return {"y": y, "state": state, "history": history}
