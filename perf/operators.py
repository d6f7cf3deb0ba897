"""The readout's operators on rows of logits, as measurable cases.

  op "top"      a teacher's record of every row: its K largest logits, their classes and the row's log-sum-exp
  op "distill"  the distillation loss of a student's rows against such records, and its gradient
  op "sample"   one class per row drawn with temperature, top-k, top-p and min-p from given uniform numbers

A row is one answer of a network: a sample's logits, the readout's membrane at one step of one sample, or one position
of a sequence model. Each operator has its plain form here, in elementary torch operations, and `own` chooses between
that and the framework's entry points. Everything is a pure function of (case, seed), made on the GPU.
"""
import math

import torch

own = False

UNIT = 2.0 ** 31  # a drawn class's weight is a whole number of 1/UNIT of the row's largest
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one batch's answers of a ten-class teacher: the smallest call, launches and host work count
        dict(name="top-readout", op="top", R=256, C=10, ld=10, dtype="f32", K=3, tau=2.0),
        # every step of a large network's readout (500 steps, 256 samples, 100 classes) recorded for a student
        dict(name="top-frames", op="top", R=128000, C=100, ld=100, dtype="f32", K=8, tau=2.0),
        # positions of a sequence teacher, an odd number of classes in padded rows
        dict(name="top-vocab", op="top", R=2048, C=32003, ld=32064, dtype="bf16", K=64, tau=1.0),
        # a few long rows in half precision
        dict(name="top-few", op="top", R=24, C=131072, ld=131072, dtype="f16", K=50, tau=1.0),
        # one batch of a ten-class student, the teacher's three listed classes taken as all of it
        dict(name="distill-readout", op="distill", R=256, C=10, ld=10, dtype="f32", K=3, tau=2.0, tail=False,
             padded=0.0),
        # every step of the large readout, the first tenth of the steps without weight
        dict(name="distill-frames", op="distill", R=128000, C=100, ld=100, dtype="f32", K=8, tau=2.0, tail=True,
             padded=0.1),
        # a sequence student in bfloat16, padded rows and padded positions
        dict(name="distill-vocab", op="distill", R=2048, C=32003, ld=32064, dtype="bf16", K=64, tau=1.0, tail=True,
             padded=0.05),
        # the longest rows, float32
        dict(name="distill-long", op="distill", R=512, C=131072, ld=131072, dtype="f32", K=32, tau=1.5, tail=False,
             padded=0.0),
        # one row's answer, the latency of a single draw
        dict(name="sample-one", op="sample", R=1, C=32003, ld=32003, dtype="f32", mix="usual"),
        # the draws of a serving batch, every request with its own settings
        dict(name="sample-serving", op="sample", R=64, C=128011, ld=128064, dtype="bf16", mix="requests"),
        # an answer at every step of a spoken-digit readout (100 steps, 256 samples, 20 classes)
        dict(name="sample-frames", op="sample", R=25600, C=20, ld=20, dtype="f32", mix="requests"),
        # many rows drawn from the whole distribution
        dict(name="sample-open", op="sample", R=1024, C=65536, ld=65536, dtype="f32", mix="open"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["top", "distill", "distill", "sample", "sample"])
    while True:
        R, C = _log(rng, 1, 131072), _log(rng, 4, 131072)
        dtype = rng.choice(["f32", "f32", "bf16", "bf16", "f16"])
        if R * C > (1 << 26) // (2 if op == "distill" and dtype == "f32" else 1):
            continue
        ld = rng.choice([C, C, -(-C // 64) * 64, C + rng.randint(1, 40)])
        case = dict(op=op, R=R, C=C, ld=ld, dtype=dtype)
        if op == "sample":
            case["mix"] = rng.choice(["usual", "requests", "requests", "open"])
        else:
            case["K"] = _log(rng, 1, min(C, 256))
            case["tau"] = rng.choice([1.0, 1.0, 1.5, 2.0, 4.0])
        if op == "distill":
            case["tail"] = rng.random() < 0.6
            case["padded"] = rng.choice([0.0, 0.0, 0.1, 0.3])
        return case


# ---------------------------------------------------------------- inputs

def _logits(case, g, spread):
    """Rows whose classes are unevenly likely, with a few strong candidates each, as trained networks give them."""
    R, C = case["R"], case["C"]
    full = torch.randn((R, case["ld"]), generator=g, device="cuda")
    full *= spread
    full += -2.0 * torch.log1p(torch.arange(case["ld"], device="cuda")[torch.randperm(case["ld"], generator=g, device="cuda")]
                               * (8.0 / C))
    n = min(C, 6)
    at = torch.randint(0, C, (R, 1), generator=g, device="cuda") + torch.arange(n, device="cuda") * (C // n)
    at %= C  # no class twice in a row
    full.scatter_(1, at, full.gather(1, at) + torch.rand((R, n), generator=g, device="cuda") * (4.0 * spread))
    return full


def _in_type(full, case):
    return full.to(DTYPES[case["dtype"]])[:, :case["C"]]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    R, C = case["R"], case["C"]
    full = _logits(case, g, 2.0)
    s = dict(case=case)
    if case["op"] == "top":
        s["logits"] = _in_type(full, case)
    elif case["op"] == "distill":
        K, tau = case["K"], case["tau"]
        teacher = full[:, :C]
        v, ids = torch.topk(teacher, K, dim=1)
        s["ids"], s["vals"] = ids.to(torch.int32), v
        s["lse"] = torch.logsumexp(teacher / tau, 1) if case["tail"] else None
        student = 0.6 * full + 0.8 * torch.randn(full.shape, generator=g, device="cuda")
        del full, teacher
        s["logits"] = _in_type(student, case)
        s["weight"] = None
        if case["padded"] > 0.0:
            live = torch.ones(R, device="cuda")
            live[:int(case["padded"] * R)] = 0.0
            s["weight"] = live / live.sum().clamp_min(1.0)
    else:
        # one class in twenty may not be answered
        out = torch.rand(C, generator=g, device="cuda") < 0.05
        out[0] = False
        full[:, :C].masked_fill_(out, -math.inf)
        s["logits"] = _in_type(full, case)
        s["u"] = torch.rand(R, generator=g, device="cuda")
        pick = torch.rand((4, R), generator=g, device="cuda")
        if case["mix"] == "usual":
            s["temperature"], s["top_k"] = torch.full((R,), 0.8, device="cuda"), torch.full((R,), 50, device="cuda")
            s["top_p"], s["min_p"] = torch.full((R,), 0.95, device="cuda"), None
        elif case["mix"] == "requests":
            s["temperature"] = torch.where(pick[0] < 0.1, torch.zeros_like(pick[0]), 0.5 + pick[0])
            s["top_k"] = torch.where(pick[1] < 0.4, torch.zeros_like(pick[1]), 1.0 + 200.0 * pick[1] ** 4)
            s["top_p"] = torch.where(pick[2] < 0.3, torch.ones_like(pick[2]), 0.5 + 0.49 * pick[2])
            s["min_p"] = torch.where(pick[3] < 0.6, torch.zeros_like(pick[3]), 0.1 * pick[3])
        else:
            s["temperature"], s["top_k"], s["top_p"], s["min_p"] = torch.ones(R, device="cuda"), None, None, None
        if s["top_k"] is not None:
            s["top_k"] = s["top_k"].to(torch.int32)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if not own:
        return {"top": _top, "distill": _distill, "sample": _sample}[op](s)
    from paper_2105_08810_amd import snn
    if op == "top":
        ids, vals, lse = snn.readout_top(s["logits"], s["case"]["K"], s["case"]["tau"])
        return dict(ids=ids, vals=vals, lse=lse)
    if op == "distill":
        loss, row_loss, grad = snn.readout_distill(s["logits"], s["ids"], s["vals"], s["lse"], s["case"]["tau"],
                                                   s["weight"])
        return dict(loss=loss, row_loss=row_loss, grad=grad)
    cls, logp, kept = snn.readout_sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    return dict(cls=cls, logp=logp, kept=kept)


def _lse(x):
    """log sum exp over a row, -inf for a row of -inf."""
    m = x.amax(1, keepdim=True)
    safe = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    return (safe + torch.log(torch.exp(x - safe).sum(1, keepdim=True)))[:, 0]


def _top(s):
    K = s["case"]["K"]
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    v, ids = torch.sort(x, dim=1, descending=True, stable=True)
    v, ids = v[:, :K], ids[:, :K].to(torch.int32)
    ids = torch.where(v == -math.inf, torch.full_like(ids, -1), ids)
    return dict(ids=ids, vals=v.contiguous(), lse=_lse(x * (1.0 / s["case"]["tau"])))


def _distill(s):
    z, ids, tau = s["logits"], s["ids"], s["case"]["tau"]
    R, C = z.shape
    x = z.float() * (1.0 / tau)
    ok = (ids >= 0) & (ids < C)
    at = torch.where(ok, ids, torch.full_like(ids, C)).long()
    none = x.new_tensor(-math.inf)
    v = torch.where(ok, s["vals"] * (1.0 / tau), none)
    if s["lse"] is not None:
        p = torch.exp(v - s["lse"][:, None])
        p_t = (1.0 - p.sum(1)).clamp_min(0.0) * (ok.sum(1) < C)
    else:
        p = torch.exp(v - torch.where(ok.any(1), _lse(v), torch.zeros_like(v[:, 0]))[:, None])
        p_t = torch.zeros_like(p[:, 0])
    mass = p.sum(1) + p_t
    member = torch.zeros((R, C + 1), dtype=torch.bool, device=z.device).scatter_(1, at, True)[:, :C]
    rest = torch.where(member, none, x)
    lse_t = _lse(rest)
    x_k = torch.where(ok, x.gather(1, at.clamp_max(C - 1)), none)
    lse = _lse(torch.cat([x_k, lse_t[:, None]], 1))
    whole = torch.where(lse == -math.inf, torch.zeros_like(lse), lse)  # a row with nothing in it: q = 0
    whole_t = torch.where(lse_t == -math.inf, torch.zeros_like(lse), lse_t)
    zero = torch.zeros_like(p_t)
    loss = torch.where(p > 0, p * (torch.log(p) - (x_k - whole[:, None])), zero[:, None]).sum(1)
    loss = loss + torch.where(p_t > 0, p_t * (torch.log(p_t) - (lse_t - whole)), zero)
    w = torch.full_like(loss, 1.0 / R) if s["weight"] is None else s["weight"]
    live = w != 0
    row_loss = torch.where(live, loss, zero)
    scale = (w * (1.0 / tau))[:, None]
    g = torch.exp(rest - whole_t[:, None]) * (scale * (mass * torch.exp(lse_t - whole) - p_t)[:, None])
    g_k = scale * (mass[:, None] * torch.exp(x_k - whole[:, None]) - p)
    g = torch.cat([g, zero[:, None]], 1).scatter_(1, at, g_k)[:, :C]
    grad = torch.where(live[:, None], g, zero[:, None]).to(z.dtype)
    return dict(loss=(w * row_loss).sum(0, keepdim=True), row_loss=row_loss, grad=grad)


def _sample(s):
    x = s["logits"].float()
    R, C = x.shape
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    m = x.amax(1, keepdim=True)
    temperature = s["temperature"][:, None]
    greedy = ~(temperature > 0)
    inv = torch.where(greedy, torch.full_like(temperature, math.inf), 1.0 / temperature)
    t = torch.where(x == m, torch.zeros_like(x), (x - m) * inv)
    e = torch.exp(t)
    n = torch.round(e * UNIT).to(torch.int64)
    _, order = torch.sort(x, dim=1, descending=True, stable=True)
    rank = torch.arange(C, device=x.device)
    ns = n.gather(1, order)
    k = torch.full_like(greedy, C, dtype=torch.int64)
    if s["top_k"] is not None:
        k = torch.where(s["top_k"][:, None] > 0, s["top_k"][:, None].long(), k)
    k = torch.where(greedy, torch.ones_like(k), k)
    ns = torch.where(rank < k, ns, torch.zeros_like(ns))
    total = ns.sum(1, keepdim=True)
    limit = total
    if s["top_p"] is not None:
        limit = torch.ceil(s["top_p"][:, None].clamp(0.0, 1.0).double() * total.double()).to(torch.int64).clamp_min(1)
    keep = (torch.cumsum(ns, 1) - ns < limit) & (ns > 0)
    if s["min_p"] is not None:
        keep &= e.gather(1, order) >= s["min_p"][:, None].clamp(0.0, 1.0)
    keep = torch.zeros_like(keep).scatter_(1, order, keep)
    keep &= m > -math.inf
    n = torch.where(keep, n, torch.zeros_like(n))
    upto = torch.cumsum(n, 1)
    total = upto[:, -1:]
    point = torch.floor(s["u"][:, None].double() * total.double()).to(torch.int64)
    point = torch.minimum(point, total - 1)
    cls = (upto <= point).sum(1)
    empty = total[:, 0] == 0
    logp = t.gather(1, cls.clamp_max(C - 1)[:, None])[:, 0] - torch.log(total[:, 0].double() / UNIT).float()
    return dict(cls=torch.where(empty, torch.full_like(cls, -1), cls).to(torch.int32),
                logp=torch.where(empty, torch.full_like(logp, -math.inf), logp), kept=keep.sum(1).to(torch.int32))


def work(case):
    R, C, size = case["R"], case["C"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "top":
        return dict(bytes=R * (C * size + 8 * case["K"] + 4), flops=3 * R * C)
    if case["op"] == "distill":
        live = R - int(case["padded"] * R)
        return dict(bytes=live * C * size + R * C * size + R * (8 * case["K"] + (12 if case["tail"] else 8)),
                    flops=6 * live * C)
    return dict(bytes=R * (C * size + 32), flops=3 * R * C)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    z = s.pop("logits").double()
    R, C = z.shape
    inf = math.inf
    if case["op"] == "top":
        return dict(ids=None, vals=torch.topk(z, case["K"], dim=1).values, lse=torch.logsumexp(z / case["tau"], 1))
    if case["op"] == "distill":
        tau, ids = case["tau"], s["ids"].long()  # every listed class is one of the row's, and none is there twice
        logq = torch.log_softmax(z / tau, 1)
        del z
        v = s["vals"].double() / tau
        if case["tail"]:
            p = torch.exp(v - s["lse"].double()[:, None])
            left = (1 - p.sum(1)).clamp_min(0) if case["K"] < C else torch.zeros_like(p[:, 0])
        else:
            p, left = torch.softmax(v, 1), torch.zeros(R, dtype=torch.float64, device=v.device)
        q = torch.exp(logq)
        others = q.scatter(1, ids, 0.0)
        out = others.sum(1)
        loss = (p * (torch.log(p) - logq.gather(1, ids))).sum(1)
        loss = loss + torch.where(left > 0, left * (torch.log(left) - torch.log(out)), torch.zeros_like(left))
        target = others * (left / out.clamp_min(1e-300))[:, None]
        target.scatter_(1, ids, p)
        w = torch.full((R,), 1.0 / R, dtype=torch.float64, device=v.device) if s["weight"] is None else s["weight"].double()
        loss = torch.where(w > 0, loss, torch.zeros_like(loss))
        grad = (q * target.sum(1, keepdim=True) - target) * (w / tau)[:, None]
        return dict(loss=(w * loss).sum(0, keepdim=True), row_loss=loss, grad=grad)
    temperature = s["temperature"].double()[:, None]
    one = temperature <= 0
    x = z / torch.where(one, torch.ones_like(temperature), temperature)
    by, order = torch.sort(x, dim=1, descending=True, stable=True)
    p = torch.softmax(by, 1)
    place = torch.arange(C, device=z.device)[None]
    keep = ~(one & (place > 0)) & (p > 0)
    if s["top_k"] is not None:
        keep &= (s["top_k"][:, None] <= 0) | (place < s["top_k"][:, None])
    p = p * keep
    p = p / p.sum(1, keepdim=True)
    if s["top_p"] is not None:
        keep &= (torch.cumsum(p, 1) - p < s["top_p"].double()[:, None]) | (place == 0)
    if s["min_p"] is not None:
        keep &= torch.exp(by - by[:, :1]) >= s["min_p"].double()[:, None]
    p = p * keep
    p = p / p.sum(1, keepdim=True)
    p = torch.zeros_like(p).scatter_(1, order, p)
    at = (torch.cumsum(p, 1) <= s["u"].double()[:, None]).sum(1, keepdim=True).clamp_max(C - 1)
    return dict(cls=None, logp=torch.log(p.gather(1, at))[:, 0], kept=None)
