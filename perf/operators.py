"""The operators on rows of class scores or logits, as they are timed and compared.

A case is a dict of plain values:

  op        "top":     the k largest logits of each row and the row's log-normalizer
            "distill": the loss against a teacher's top logits, and its gradient
            "sample":  a class per row by temperature, top-k, top-p and min-p from
                       given Gumbel numbers
  rows, classes, k       k: entries of the top list (for "sample": the top-k, 0 none)
  type      "int32" (scores), "float32", "float16" or "bfloat16"
  pad       elements between the end of a row and the next one's start
  mode      top: ""; distill: "both" (loss and gradient in one call), "loss"
            (evaluation) or "autograd" (a differentiable loss, then its backward
            pass); sample: "one" (the same parameters for all rows) or "each" (a
            request's own parameters per row, of every kind)
  rest      distill: whether the teacher's log-normalizer is known, so that the mass
            outside its list counts
  temperature, top_p, min_p

Rows of 10 to 100 classes are those of this library's networks; longer ones are
vocabularies and label sets in general.
"""
import math

import torch

own = False
DEVICE = "cuda"
TYPES = {"int32": torch.int32, "float32": torch.float32, "float16": torch.float16,
         "bfloat16": torch.bfloat16}
BYTES = {"int32": 4, "float32": 4, "float16": 2, "bfloat16": 2}
LARGEST = 2048 * 131072          # elements of the largest listed case


def _case(name, op, rows, classes, k, type_, mode="", temperature=1.0, rest=False, top_p=1.0,
          min_p=0.0, pad=0):
    return {"name": name, "op": op, "rows": rows, "classes": classes, "k": k, "type": type_,
            "mode": mode, "temperature": temperature, "rest": rest, "top_p": top_p,
            "min_p": min_p, "pad": pad}


def listed():
    return [
        # one item's teacher list asked for by itself: latency
        _case("top_one", "top", 1, 50021, 256, "float32"),
        # the scores of the widest network's whole batch, kept as a teacher's lists
        _case("top_scores", "top", 1 << 18, 100, 10, "int32", temperature=20.0),
        # a teacher's lists over a training batch of tokens, the largest read
        _case("top_vocab", "top", 2048, 131072, 64, "bfloat16"),
        # the head of a 100-class network fitted to a wider one's lists, a whole batch
        _case("distill_head", "distill", 1 << 18, 100, 10, "float32", "both", 2.0, True),
        # a training step over tokens, padding rows among them
        _case("distill_vocab", "distill", 4096, 65536, 64, "bfloat16", "both", 2.0, True),
        # the same through autograd at odd sizes in float16, teacher cut to its list
        _case("distill_ragged", "distill", 1021, 50021, 33, "float16", "autograd", 1.5),
        # held-out loss, no gradient
        _case("distill_eval", "distill", 4099, 32003, 20, "bfloat16", "loss", 1.0, True),
        # labels drawn from the smallest network's scores for one packed word of samples
        _case("sample_scores", "sample", 64, 10, 0, "int32", "one", 8.0),
        # one request's next token
        _case("sample_one", "sample", 1, 131072, 50, "bfloat16", "one", 0.8, top_p=0.95),
        # a serving batch in which every request has parameters of its own
        _case("sample_batch", "sample", 256, 131072, 50, "bfloat16", "each", 0.8, top_p=0.9,
              min_p=0.02),
        # nucleus sampling alone over odd rows
        _case("sample_nucleus", "sample", 509, 32003, 0, "float16", "one", 0.9, top_p=0.9),
        # plain sampling by temperature: every class and every number counts
        _case("sample_plain", "sample", 1024, 50021, 0, "float32", "one", 0.7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["top", "distill", "distill", "sample", "sample"])
        classes = _log_int(rng, 10, 131072)
        if rng.random() < 0.25:
            classes = rng.choice([10, 11, 37, 100, 32768, 65536, 131072])
        rows = _log_int(rng, 1, 1 << 18)
        if rows * classes * (2 if op == "distill" else 1) > LARGEST // 2:
            continue
        c = _case("", op, rows, classes, 0, rng.choice(["float32", "float16", "bfloat16"]),
                  pad=rng.choice([0, 0, 0, rng.randint(1, 64)]))
        del c["name"]
        if op != "distill" and classes <= 4096 and rng.random() < 0.3:
            c["type"] = "int32"
        c["temperature"] = round(rng.uniform(5.0, 40.0) if c["type"] == "int32"
                                 else rng.uniform(0.5, 2.0), 2)
        if op == "top":
            c["k"] = min(classes, _log_int(rng, 1, 1024))
        elif op == "distill":
            c["k"] = min(classes, _log_int(rng, 1, 256))
            c["mode"] = rng.choice(["both", "both", "loss", "autograd"])
            c["rest"] = rng.random() < 0.5 and c["k"] < classes
        else:
            c["mode"] = rng.choice(["one", "one", "each"])
            if rng.random() < 0.5:
                c["k"] = min(classes, _log_int(rng, 1, 1024))
            if rng.random() < 0.5:
                c["top_p"] = round(rng.uniform(0.5, 0.99), 2)
            if rng.random() < 0.3:
                c["min_p"] = round(rng.uniform(0.005, 0.2), 3)
        return c


def _strided(x, pad):
    """x with `pad` unused elements after each row."""
    if not pad:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=DEVICE)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _spread(n, c, k, gen):
    """k distinct classes of each row."""
    step = max(1, int(0.618 * c / k))
    first = torch.randint(0, c, (n, 1), device=DEVICE, generator=gen)
    return (first + step * torch.arange(k, device=DEVICE)) % c


def _logits(case, gen):
    """Scores of a network's classes, or logits of a vocabulary: a common falling
    slope over shuffled classes, noise, and a few likely classes per row."""
    n, c = case["rows"], case["classes"]
    x = torch.randn((n, c), device=DEVICE, generator=gen)
    likely = _spread(n, c, 6, gen)
    lift = 2 + 2 * torch.randn((n, 6), device=DEVICE, generator=gen).abs()
    if case["type"] == "int32":        # ones among a class's 640 nodes
        x.mul_(12.6).add_(320).scatter_add_(1, likely, 24 * lift)
        return x.round_().clamp_(0, 640).to(torch.int32)
    slope = torch.log1p(torch.randperm(c, device=DEVICE, generator=gen).float())
    x.mul_(1.5).sub_(slope).scatter_add_(1, likely, lift + 0.75 * math.log(c))
    return x.to(TYPES[case["type"]])


def prepare(case, seed):
    gen = torch.Generator(DEVICE)
    gen.manual_seed(int(seed))
    n, c, k = case["rows"], case["classes"], case["k"]
    s = {"case": case, "logits": _logits(case, gen)}
    if case["op"] == "distill":
        # a list of k distinct classes a row, falling values, and the student's logits
        # raised at most of them
        at = _spread(n, c, k, gen)
        values = 6 * torch.rand((n, k), device=DEVICE, generator=gen) ** 2 + 4
        values = values.sort(dim=1, descending=True).values
        raised = values + 1.5 * torch.randn((n, k), device=DEVICE, generator=gen)
        s["logits"].scatter_(1, at, raised.to(s["logits"].dtype))
        s["top_values"], s["top_indices"] = values.to(s["logits"].dtype), at.to(torch.int32)
        s["top_log_norm"] = None
        if case["rest"]:
            inside = torch.logsumexp(s["top_values"].float() / case["temperature"], 1)
            share = 0.6 + 0.38 * torch.rand((n,), device=DEVICE, generator=gen)
            s["top_log_norm"] = inside - torch.log(share)
        # a mean over the rows that count: one in eight is padding
        counts = torch.rand((n,), device=DEVICE, generator=gen) > 0.125
        s["weight"] = counts.float() * case["temperature"] ** 2
        if case["mode"] == "autograd":
            s["logits"] = _strided(s["logits"], case["pad"]).detach().requires_grad_()
    if case["op"] == "sample":
        # standard Gumbel numbers, -log(-log u)
        g = torch.empty((n, c), device=DEVICE).exponential_(generator=gen)
        s["noise"] = g.log_().neg_()
        kinds = torch.randint(0, 4, (n,), device=DEVICE, generator=gen)
        each = case["mode"] == "each"
        s["temperature"], s["top_k"] = case["temperature"], k
        s["top_p"], s["min_p"] = case["top_p"], case["min_p"]
        if each:      # greedy rows, rows without a filter, and every mixture of filters
            wide = 0.5 + torch.rand((n,), device=DEVICE, generator=gen)
            s["temperature"] = torch.where(kinds == 0, 0.0, wide * case["temperature"])
            s["top_k"] = torch.where(kinds != 1, k, 0).to(torch.int32)
            s["top_p"] = torch.where(kinds != 2, case["top_p"], 1.0).float()
            s["min_p"] = torch.where(kinds == 3, case["min_p"], 0.0).float()
    if not s["logits"].requires_grad:
        s["logits"] = _strided(s["logits"], case["pad"])
    return s


# ---------------------------------------------------------------- plain forms

def _top(s, case):
    x = s["logits"]
    values, indices = torch.sort(x, dim=1, descending=True, stable=True)
    y = x.float() * (1 / case["temperature"])
    m = y.max(1, keepdim=True).values
    log_norm = m[:, 0] + torch.log(torch.exp(y - m).sum(1))
    k = case["k"]
    return values[:, :k].contiguous(), indices[:, :k].to(torch.int32), log_norm


def _distill(s, case, weight, want_loss, want_grad):
    scale = 1 / case["temperature"]
    y = s["logits"].detach().float() * scale
    at = s["top_indices"].long()
    t = s["top_values"].float() * scale
    if s["top_log_norm"] is None:
        mt = t.max(1, keepdim=True).values
        log_q = t - mt - torch.log(torch.exp(t - mt).sum(1, keepdim=True))
    else:
        log_q = t - s["top_log_norm"][:, None]
    q = torch.exp(log_q)
    m = y.max(1, keepdim=True).values
    e = torch.exp(y - m)
    total = e.sum(1, keepdim=True)
    loss = grad = None
    e_rest = e.scatter(1, at, 0.0) if case["rest"] else None
    if case["rest"]:
        rest = e_rest.sum(1, keepdim=True)
        q_rest = (1 - q.sum(1, keepdim=True)).clamp(min=0)
    if want_loss:
        log_p = y.gather(1, at) - m - torch.log(total)
        loss = (q * (log_q - log_p)).sum(1)
        if case["rest"]:
            loss = loss + (q_rest * (torch.log(q_rest) - torch.log(rest / total)))[:, 0]
        loss = loss * weight
    if want_grad:
        if case["rest"]:
            grad = e_rest * (1 / total - q_rest / rest)
            grad.scatter_(1, at, e.gather(1, at) / total - q)
        else:
            grad = e * (q.sum(1, keepdim=True) / total)
            grad.scatter_add_(1, at, -q)
        grad = (grad * (weight * scale)[:, None]).to(s["logits"].dtype)
    return loss, grad


def _sample(s, case):
    x = s["logits"]
    n, c = x.shape
    column = lambda v: (v.reshape(-1, 1) if torch.is_tensor(v)            # noqa: E731
                        else torch.full((1, 1), v, device=DEVICE))
    temperature, top_k = column(s["temperature"]).float(), column(s["top_k"])
    top_p, min_p = column(s["top_p"]).float(), column(s["min_p"]).float()
    ordered, order = torch.sort(x, dim=1, descending=True, stable=True)
    ordered = ordered.float()
    greedy = temperature <= 0
    inverse = 1 / torch.where(greedy, 1.0, temperature)
    y = (ordered - ordered[:, :1]) * inverse
    rank = torch.arange(c, device=DEVICE)
    keep = (rank < torch.where(top_k > 0, top_k, c)) & (~greedy | (rank == 0))
    e = torch.where(keep, torch.exp(y), 0.0)
    before = torch.cumsum(e, 1) - e
    keep = keep & ((top_p >= 1) | (rank == 0) | (before < top_p * e.sum(1, keepdim=True)))
    keep = keep & ((min_p <= 0) | (y >= torch.log(min_p)))
    score = torch.where(keep, y + s["noise"].gather(1, order), -math.inf)
    best = score == score.max(1, keepdim=True).values
    token = torch.where(best, order, c).min(1).values
    chosen = torch.where(order == token[:, None], y, 0.0).sum(1)
    log_prob = chosen - torch.log(torch.where(keep, e, 0.0).sum(1))
    return token.to(torch.int32), log_prob


def run(s):
    case = s["case"]
    if own:
        from paper_2602_07400_amd import bitlogic as bl
    if case["op"] == "top":
        if own:
            return bl.bitlogic_top_logits(s["logits"], case["k"], temperature=case["temperature"])
        return _top(s, case)
    if case["op"] == "sample":
        if own:
            return bl.bitlogic_sample(s["logits"], s["noise"], temperature=s["temperature"],
                                      top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return _sample(s, case)
    if case["mode"] == "autograd":
        if own:
            loss = bl.bitlogic_distill_loss(s["logits"], s["top_values"], s["top_indices"],
                                            s["top_log_norm"], temperature=case["temperature"],
                                            top_temperature=case["temperature"])
            grad, = torch.autograd.grad(loss, s["logits"], s["weight"])
            return loss.detach(), grad
        loss, _ = _distill(s, case, torch.ones_like(s["weight"]), True, False)
        _, grad = _distill(s, case, s["weight"], False, True)
        return loss, grad
    grads = case["mode"] == "both"
    if own:
        return bl.bitlogic_distill(s["logits"], s["top_values"], s["top_indices"],
                                   s["top_log_norm"], temperature=case["temperature"],
                                   top_temperature=case["temperature"], row_weight=s["weight"],
                                   want_grad=grads)
    return _distill(s, case, s["weight"], True, grads)


def work(case):
    n, c, k, b = case["rows"], case["classes"], case["k"], BYTES[case["type"]]
    elements = n * c
    if case["op"] == "top":              # logits once; values, indices, log-normalizer
        return {"bytes": elements * b + n * (k * (b + 4) + 4), "flops": 4 * elements}
    if case["op"] == "distill":
        passes = {"both": 2, "loss": 1, "autograd": 3}[case["mode"]]   # autograd reads twice
        lists = n * (k * (b + 4) + (4 if case["rest"] else 0)) * (2 if passes == 3 else 1)
        return {"bytes": elements * b * passes + lists + 8 * n,
                "flops": (4 if passes == 1 else 8) * elements}
    # the kept classes' numbers; how many a top-p keeps depends on the logits
    filtered = k > 0 or case["top_p"] < 1 or case["min_p"] > 0
    numbers = n * min(c, k) if filtered else elements
    return {"bytes": elements * b + 4 * numbers + 8 * n, "flops": 4 * elements}


# ------------------------------------------------- 64 bits, from the definitions

def _exact_top(s, case, rows):
    x = s["logits"][rows].double()
    # the order as one key: descending value, then ascending class
    order = torch.argsort(-x, dim=1, stable=True)[:, :case["k"]]
    return (x.gather(1, order), None, torch.logsumexp(x / case["temperature"], 1))


def _exact_distill(s, case, rows):
    t = case["temperature"]
    at = s["top_indices"][rows].long()
    log_p = torch.log_softmax(s["logits"][rows].detach().double() / t, 1)
    teacher = s["top_values"][rows].double() / t
    if s["top_log_norm"] is None:
        log_q = torch.log_softmax(teacher, 1)
    else:
        log_q = teacher - s["top_log_norm"][rows].double()[:, None]
    q = log_q.exp()
    w = s["weight"][rows].double()
    # d loss / d log p_i, then through the log-softmax: g - p * sum g
    g = torch.zeros_like(log_p).scatter_(1, at, -q)
    loss = (q * (log_q - log_p.gather(1, at))).sum(1)
    if case["rest"]:
        q_rest = 1 - q.sum(1)
        outside = log_p.scatter(1, at, -math.inf)
        log_rest = torch.logsumexp(outside, 1)
        loss = loss + q_rest * (q_rest.log() - log_rest)
        g = g - q_rest[:, None] * (outside - log_rest[:, None]).exp()
    grad = (g - log_p.exp() * g.sum(1, keepdim=True)) * (w / t)[:, None]
    return (loss if case["mode"] == "autograd" else loss * w,
            None if case["mode"] == "loss" else grad)


def _exact_sample(s, case, rows):
    x = s["logits"][rows].double()
    n, c = x.shape
    of = lambda v: (v[rows].double() if torch.is_tensor(v)                 # noqa: E731
                    else torch.full((n,), float(v), device=DEVICE, dtype=torch.float64))
    t, k, p, floor = (of(s[name])[:, None] for name in ("temperature", "top_k", "top_p", "min_p"))
    y = torch.where(t > 0, (x - x.max(1, keepdim=True).values) / t.clamp(min=1e-30), 0.0)
    order = torch.argsort(-x, dim=1, stable=True)
    place = torch.empty_like(order).scatter_(1, order,
                                             torch.arange(c, device=DEVICE).expand(n, c))
    kept = (place == 0) | ((t > 0) & ((k <= 0) | (place < k)))
    mass = y.exp() * kept
    sums = mass.gather(1, order).cumsum(1)
    share = sums.gather(1, place) - mass          # of the classes before, in the order
    kept = kept & ((place == 0) | (p >= 1) | (share < p * mass.sum(1, keepdim=True)))
    kept = kept & ((floor <= 0) | (y.exp() >= floor))
    score = torch.where(kept, y + s["noise"][rows].double(), -math.inf)
    token = score.argmax(1, keepdim=True)
    return None, (y.gather(1, token)[:, 0] - (y.exp() * kept).sum(1).log())


def exact(case, seed):
    s = prepare(case, seed)
    if s["logits"].requires_grad:
        s["logits"] = s["logits"].detach()
    of = {"top": _exact_top, "distill": _exact_distill, "sample": _exact_sample}[case["op"]]
    parts = []
    step = max(1, (1 << 25) // case["classes"])
    for first in range(0, case["rows"], step):
        parts.append(of(s, case, slice(first, min(case["rows"], first + step))))
    return tuple(None if p[0] is None else torch.cat(p) for p in zip(*parts))
