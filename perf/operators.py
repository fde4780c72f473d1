"""What the speed of the operators on rows of logits is measured on.

A row holds one logit (or Q-value) per action.  Three operators work on such rows: choosing an
action from given random numbers (temperature, top-k, top-p, min-p), a teacher's top actions with
the row's log-sum-exp, and the loss that distils them into a student, with its gradient.

Kinds of cases
  choose  one action per row; outputs: its index and its log-probability
  top     the k largest logits of every row; outputs: values, indices, log-sum-exp
  loss    distillation loss of every row
  grad    distillation loss of every row and the gradient of the student's logits

The action sets are those of the benchmark and the tests (30 actions, rows in a table of pitch 32
as the trainer keeps them) and generic ones up to those of a vocabulary.
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _choose(**kw):
    # filter: "none" (temperature alone), "k" (top-k), "p" (top-p and min-p), "mixed" (every row its own)
    return {"kind": "choose", "dtype": "f32", "rows": 1, "n": 30, "pad": 0, "sigma": 1.0, "masked": 0.0,
            "filter": "none", **kw}


def _top(**kw):
    return {"kind": "top", "dtype": "f32", "rows": 1, "n": 30, "pad": 0, "sigma": 1.0, "masked": 0.0, "k": 8, **kw}


def _distill(kind, **kw):
    # rest: the teacher's mass outside its top logits counts as one bin; idle: share of rows of weight 0
    return {"kind": kind, "dtype": "f32", "rows": 1, "n": 30, "pad": 0, "sigma": 1.0, "k": 8, "rest": False,
            "idle": 0.0, **kw}


def listed():
    return [
        # One actor asks for its next action: the smallest call, the loop of acting and learning.
        _choose(name="choose_1x30"),
        # A batch of actors over the trainer's own table of Q-values, some actions not allowed,
        # every actor with its own exploration.
        _choose(name="choose_128x30_mixed", rows=128, pad=2, masked=0.1, filter="mixed"),
        # One sequence's next token from a large vocabulary, top-k: a single row.
        _choose(name="choose_1x131072_topk", dtype="bf16", n=131_072, sigma=2.5, filter="k"),
        # Some sequences in full precision, the nucleus cut from an odd number of actions.
        _choose(name="choose_37x50021_topp", rows=37, n=50_021, sigma=2.0, filter="p"),
        # A full serving batch, every request with its own settings: the largest choice.
        _choose(name="choose_256x131072_mixed", dtype="bf16", rows=256, n=131_072, sigma=2.5, filter="mixed"),
        # A teacher writes down the best actions of a batch.
        _top(name="top_128x30_k8", rows=128, pad=2),
        # A teacher's top logits over a vocabulary for many tokens.
        _top(name="top_2048x32768_k64", dtype="bf16", rows=2048, n=32_768, sigma=2.5, k=64),
        # Few rows, odd length, many entries, in full precision.
        _top(name="top_9x100003_k500", rows=9, n=100_003, sigma=2.0, masked=0.05, k=500),
        # A student learns a batch of action rows.
        _distill("grad", name="grad_128x30_k8", rows=128, pad=2, rest=True),
        # The training step over a vocabulary: the largest case.
        _distill("grad", name="grad_4096x32768_k64", dtype="bf16", rows=4096, n=32_768, sigma=2.5, k=64, rest=True,
                 idle=0.1),
        # Few long rows in full precision, the teacher's entries renormalised.
        _distill("grad", name="grad_11x131071_k300", rows=11, n=131_071, sigma=2.0, k=300),
        # A student's loss on held-out rows, without a gradient.
        _distill("loss", name="loss_1000x50021_k32", dtype="bf16", rows=1000, n=50_021, sigma=2.0, k=32, rest=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["choose", "choose", "choose", "top", "top", "grad", "grad", "loss"])
    most = {"choose": 2 ** 25, "top": 2 ** 26, "grad": 2 ** 27, "loss": 2 ** 27}[kind]
    n = _log_int(rng, 2, 160_000)
    case = {"dtype": rng.choice(["f32", "bf16"]), "n": n, "rows": _log_int(rng, 1, max(1, min(4096, most // n))),
            "pad": rng.choice([0, 0, 1, 2, 8]), "sigma": round(rng.uniform(0.5, 3.0), 2)}
    if case["dtype"] == "f32":
        case["rows"] = max(1, case["rows"] // 2)
    if kind == "choose":
        return _choose(masked=rng.choice([0.0, 0.0, 0.3]), filter=rng.choice(["none", "k", "p", "mixed"]), **case)
    case["k"] = _log_int(rng, 1, min(n, 1000))
    if kind == "top":
        return _top(masked=rng.choice([0.0, 0.2]), **case)
    return _distill(kind, rest=rng.random() < 0.5, idle=rng.choice([0.0, 0.2]), **case)


# ------------------------------------------------------------------------------------- inputs
def _live(case):
    """Rows that count: the others stand at the end of the batch, as padding does."""
    return case["rows"] - int(case["rows"] * case.get("idle", 0.0))


def _logits(case, gen):
    """rows x n logits in a table with `pad` more columns: normal deviates, a few actions well above the
    rest, and a share of actions that are not allowed."""
    rows, n = case["rows"], case["n"]
    x = torch.randn((rows, n), device="cuda", generator=gen).mul_(case["sigma"])
    few = min(n, 16)
    liked = torch.randint(0, n, (rows, 1), device="cuda", generator=gen)
    liked = (liked + torch.arange(few, device="cuda") * (n // few)) % n
    x.scatter_add_(1, liked, torch.rand((rows, few), device="cuda", generator=gen) * (2 * case["sigma"]))
    if case.get("masked"):
        x.masked_fill_(torch.rand((rows, n), device="cuda", generator=gen) < case["masked"], -math.inf)
    table = torch.zeros((rows, n + case["pad"]), dtype=_DTYPE[case["dtype"]], device="cuda")
    table[:, :n] = x
    return table[:, :n], x


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows, n, kind = case["rows"], case["n"], case["kind"]
    logits, x = _logits(case, gen)
    state = {"kind": kind, "logits": logits}

    def pick(values, dtype=torch.float32):
        at = torch.randint(0, len(values), (rows,), device="cuda", generator=gen)
        return torch.tensor(values, dtype=dtype, device="cuda")[at]

    if kind == "choose":
        state["u"] = torch.rand(rows, device="cuda", generator=gen)
        state["how"] = {
            "none": lambda: {"temperature": 0.8},
            "k": lambda: {"temperature": 0.8, "top_k": 50},
            "p": lambda: {"top_p": 0.9, "min_p": 0.002},
            "mixed": lambda: {"temperature": pick([0.0, 0.6, 0.8, 1.0, 1.0, 1.3]),
                              "top_k": pick([0, 0, 5, 20, 50, 200], torch.int32),
                              "top_p": pick([0.5, 0.9, 0.95, 1.0, 1.0]), "min_p": pick([0.0, 0.0, 0.01, 0.1])},
        }[case["filter"]]()
        return state
    k = min(case["k"], n)
    state["k"] = k
    if kind == "top":
        state["temperature"] = 1.0
        return state
    # the teacher agrees with the student in part
    t = x.mul_(0.7)
    t += torch.randn((rows, n), device="cuda", generator=gen).mul_(0.7 * case["sigma"])
    t = t.to(_DTYPE[case["dtype"]]).float()
    state["teacher_temperature"], state["student_temperature"] = 0.9, 1.1
    top = torch.topk(t, k, dim=1)
    state["teacher"], state["index"] = top.values.to(_DTYPE[case["dtype"]]), top.indices.to(torch.int32)
    state["rest"] = torch.logsumexp(t / state["teacher_temperature"], dim=1) if case["rest"] else None
    if k > 2:    # a part of the rows has fewer entries
        short = torch.rand(rows, device="cuda", generator=gen) < 0.2
        state["index"][short, k - 1] = -1
    state["weight"] = torch.rand(rows, device="cuda", generator=gen).add_(0.5).div_(rows)
    state["weight"][_live(case):] = 0.0
    return state


# ------------------------------------------------------------------------------- the plain forms
def _column(v, like):
    return v.to(like.dtype)[:, None] if torch.is_tensor(v) else torch.full_like(like, v)


def _plain_choose(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    # in 64 bits: a sum's last bits decide between two actions where u falls next to a border
    n = logits.shape[1]
    v, order = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    allowed = v > -math.inf
    v = v.double()
    first = v[:, :1]
    T, K, P, least = (_column(a, first) for a in (temperature, top_k, top_p, min_p))
    greedy = ~(T > 0)
    w = torch.where(allowed, torch.exp((v - first) / torch.where(greedy, 1.0, T)), 0.0)
    place = torch.arange(n, device=v.device)[None, :]
    in_k = place < torch.where((K > 0) & (K < n), K, float(n))
    w = torch.where(in_k, w, 0.0)
    c = torch.cumsum(w, dim=1)
    before = torch.cat([torch.zeros_like(first), c[:, :-1]], dim=1)
    keep = allowed & in_k & ((before < P * c[:, -1:]) | ~(P < 1)) & ((w >= least) | ~(least > 0))
    keep = torch.where(greedy, False, keep)
    keep[:, 0] = allowed[:, 0]
    kept = keep.sum(dim=1, keepdim=True)
    last = (kept - 1).clamp(min=0)
    mass = torch.gather(c, 1, last)
    at = torch.minimum((c <= u.double()[:, None] * mass).sum(dim=1, keepdim=True), last)
    index = torch.where(kept > 0, torch.gather(order, 1, at), -1)
    logp = torch.where((kept > 0) & ~greedy, torch.log(torch.gather(w, 1, at) / mass), 0.0)
    return index[:, 0].to(torch.int32), logp[:, 0].float()


def _plain_exp(z, temperature):
    """exp((z - max) / temperature), its sum over each row in 64 bits, and the row's log-sum-exp."""
    m = z.amax(dim=1, keepdim=True)
    m = torch.where(m > -math.inf, m, 0.0)
    e = torch.exp((z - m) / temperature)
    total = e.sum(dim=1, keepdim=True, dtype=torch.float64)
    return e, total, m.double() / temperature + torch.log(total)


def _plain_top(logits, k, temperature):
    v, order = torch.sort(logits, dim=1, descending=True, stable=True)
    lse = _plain_exp(logits.float(), temperature)[2]
    v = v[:, :k].contiguous()
    return v, torch.where(v > -math.inf, order[:, :k], -1).to(torch.int32), lse[:, 0].float()


def _plain_distill(logits, teacher, index, weight, student_temperature, teacher_temperature, teacher_lse, gradient):
    # What is summed over a row or made of the entries alone is held in 64 bits: the loss is a small
    # difference of large logarithms.
    z = logits.float()
    there = (index >= 0) & (index < z.shape[1])
    at = torch.where(there, index, 0).long()
    t = torch.where(there, teacher.double() / teacher_temperature, -math.inf)
    log_q = t - (_plain_exp(t, 1.0)[2] if teacher_lse is None else teacher_lse.double()[:, None])
    q = torch.exp(log_q)
    sum_q = q.sum(dim=1, keepdim=True)
    e, total, lse = _plain_exp(z, student_temperature)
    log_p = torch.where(there, torch.gather(z, 1, at).double() / student_temperature - lse, -math.inf)
    p = torch.exp(log_p)
    loss = torch.where(q > 0, q * (log_q - log_p), 0.0).sum(dim=1, keepdim=True)
    inside = outside = sum_q          # what p_i is multiplied by in the gradient
    if teacher_lse is not None:
        named = torch.zeros(z.shape, dtype=torch.int32, device=z.device).scatter_add_(1, at, there.to(torch.int32)) > 0
        p_rest = torch.where(named, 0.0, e).sum(dim=1, keepdim=True, dtype=torch.float64) / total
        sum_p = p.sum(dim=1, keepdim=True)
        rest = (sum_q < 1) & (p_rest > 0)
        log_p_rest = torch.where(sum_p < 0.5, torch.log1p(-sum_p), torch.log(p_rest))
        loss = loss + torch.where(rest, (1 - sum_q) * (torch.log1p(-sum_q) - log_p_rest), 0.0)
        inside = torch.where(rest, 1.0, sum_q)
        outside = torch.where(rest, (sum_q - sum_p) / p_rest, sum_q)
    live = (weight != 0)[:, None]
    loss = torch.where(live, loss * weight[:, None], 0.0)[:, 0].float()
    if not gradient:
        return loss
    scale = weight.double()[:, None] / student_temperature
    g = e * torch.where(live, scale * outside / total, 0.0).float()
    g.scatter_add_(1, at, torch.where(there & live, scale * (p * (inside - outside) - q), 0.0).float())
    return loss, torch.where(live, g, 0.0).to(logits.dtype)


# --------------------------------------------------------------------------------- one pass
def run(state):
    kind, logits = state["kind"], state["logits"]
    if kind == "choose":
        if own:
            from paper_1801_03138_amd import binding as B
            return B.choose_actions(logits, state["u"], **state["how"])
        return _plain_choose(logits, state["u"], **state["how"])
    if kind == "top":
        if own:
            from paper_1801_03138_amd import binding as B
            return B.top_actions(logits, state["k"], temperature=state["temperature"])
        return _plain_top(logits, state["k"], state["temperature"])
    if own:
        from paper_1801_03138_amd import binding as B
        call = B.distill_grad if kind == "grad" else B.distill_loss
        return call(logits, state["teacher"], state["index"], weight=state["weight"], teacher_lse=state["rest"],
                    student_temperature=state["student_temperature"],
                    teacher_temperature=state["teacher_temperature"])
    return _plain_distill(logits, state["teacher"], state["index"], state["weight"], state["student_temperature"],
                          state["teacher_temperature"], state["rest"], kind == "grad")


# ----------------------------------------------------------------------- the definition in 64 bits
def _value(v, row):
    return float(v[row]) if torch.is_tensor(v) else float(v)


def _exact_choose(state, case):
    how, u = state["how"], state["u"].double().cpu()
    x = state["logits"].double()
    logp, index = [], []
    for row in range(case["rows"]):
        a = x[row]
        ids = torch.nonzero(a > -math.inf)[:, 0]
        T, K = _value(how.get("temperature", 1.0), row), int(_value(how.get("top_k", 0), row))
        P, least = _value(how.get("top_p", 1.0), row), _value(how.get("min_p", 0.0), row)
        if not len(ids):
            index.append(-1)
            logp.append(0.0)
            continue
        ids = ids[torch.argsort(-a[ids], stable=True)]
        if K > 0:
            ids = ids[:K]
        if not T > 0:
            ids = ids[:1]
            T = 1.0
        w = torch.exp(a[ids] / T - a[ids[0]] / T)
        share = torch.cumsum(w / w.sum(), 0) - w / w.sum()
        count = len(ids)
        if P < 1:
            count = min(count, int((share < P).sum()))
        if least > 0:
            count = min(count, int((w >= least).sum()))
        w = w[:max(count, 1)]
        w = w / w.sum()
        at = min(int((torch.cumsum(w, 0) <= u[row]).sum()), len(w) - 1)
        index.append(int(ids[at]))
        logp.append(math.log(float(w[at])))
    return torch.tensor(index, dtype=torch.int32), torch.tensor(logp, dtype=torch.float64)


def _exact_distill(state, case):
    logits, gradient = state["logits"], case["kind"] == "grad"
    rows, n = logits.shape
    weight, ts = state["weight"].double(), state["student_temperature"]
    piece = max(1, 2 ** 25 // n)
    loss = torch.zeros(rows, dtype=torch.float64, device=logits.device)
    out = torch.zeros((rows, n), dtype=torch.float64, device=logits.device) if gradient else None
    for lo in range(0, _live(case), piece):
        s = slice(lo, min(lo + piece, _live(case)))
        log_p = torch.log_softmax(logits[s].double() / ts, dim=1)
        index = state["index"][s].long()
        gone = index < 0
        t = (state["teacher"][s].double() / state["teacher_temperature"]).masked_fill(gone, -math.inf)
        log_q = t - state["rest"][s].double()[:, None] if case["rest"] else torch.log_softmax(t, dim=1)
        # one more column takes the entries that are not there
        target = torch.zeros((log_p.shape[0], n + 1), dtype=torch.float64, device=logits.device)
        target.scatter_(1, index.masked_fill(gone, n), log_q.exp().masked_fill(gone, 0.0))
        target = target[:, :n]
        named = torch.zeros((log_p.shape[0], n + 1), dtype=torch.bool, device=logits.device)
        named = named.scatter_(1, index.masked_fill(gone, n), True)[:, :n]
        value = torch.where(target > 0, target * (torch.log(target) - log_p), 0.0).sum(1)
        if case["rest"]:
            left = (1.0 - target.sum(1)).clamp(min=0.0)
            p_rest = log_p.exp().masked_fill(named, 0.0).sum(1)
            left = torch.where(p_rest > 0, left, 0.0)
            value = value + torch.where(left > 0, left * (torch.log(left) - torch.log(p_rest)), 0.0)
            share = torch.where(p_rest > 0, left / p_rest, 0.0)
            if gradient:
                target = torch.where(named, target, log_p.exp() * share[:, None])
        loss[s] = value * weight[s]
        if gradient:
            g = log_p.exp() * target.sum(1, keepdim=True) - target
            out[s] = g * (weight[s] / ts)[:, None]
    return (loss, out) if gradient else loss


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "choose":
        return _exact_choose(state, case)
    if case["kind"] == "top":
        x = state["logits"].double()
        index = torch.argsort(-x, dim=1, stable=True)[:, :state["k"]]
        value = torch.gather(x, 1, index)
        return (value, torch.where(value > -math.inf, index, -1).to(torch.int32),
                torch.logsumexp(x / state["temperature"], dim=1))
    return _exact_distill(state, case)


# ------------------------------------------------------------- what a pass cannot do without
def work(case):
    rows, n, e, kind = case["rows"], case["n"], _BYTES[case["dtype"]], case["kind"]
    if kind == "choose":
        # the logits and a random number in, an index and a log-probability out; difference, scale, exp, sum
        settings = 16 if case["filter"] == "mixed" else 0
        return {"bytes": rows * (n * e + 12 + settings), "flops": 4 * rows * n}
    k = min(case["k"], n)
    if kind == "top":
        return {"bytes": rows * (n * e + k * (e + 4) + 4), "flops": 4 * rows * n}
    live = _live(case)
    entries = live * k * (e + 4) + rows * 8 + (4 * live if case["rest"] else 0)
    if kind == "loss":
        return {"bytes": live * n * e + entries, "flops": 4 * live * n}
    return {"bytes": (live + rows) * n * e + entries, "flops": 8 * live * n}
