"""Operators on rows of logits and of probabilities, as measurable cases.

Kinds of work (field "op"):

top      the largest logits of every row, with their words and the row's log-sum-exp: a teacher's lists for distillation, the top
         words of a topic, the candidates of a decoding step.
distill  the loss of a student against a teacher's top logits, tau^2 KL(teacher || student) per row, either over the listed
         words alone or (tail) with one bucket more for all that the list leaves out; with "grad", the loss and its gradient
         with respect to the student's logits, as a training step needs them.
verify   drafted tokens against the target's probabilities: the leading drafts that the test u q < p accepts, then one more token,
         drawn from max(p - q, 0) at the first refusal or from p behind the last draft.

Vocabularies and topic counts of the listed cases are those of synth.CONFIGS and the library's limit of K, beside odd ones.
`pad` is what a row's stride has over its length.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZES = {"float32": 4, "float16": 2, "bfloat16": 2}
MASS = 42          # probabilities are held as multiples of 2^-42 where a token is drawn
TOP_MOST = 512     # longest list


def _top(name, rows, V, top, dtype, pad=0, masked=False, tau=1.0):
    c = dict(op="top", rows=rows, V=V, pad=pad, top=top, dtype=dtype, tau=tau, masked=masked)
    return dict(c, name=name) if name else c


def _distill(name, rows, V, top, dtype, tail, grad, pad=0, masked=False, tau=1.0):
    c = dict(op="distill", rows=rows, V=V, pad=pad, top=top, dtype=dtype, tail=tail, grad=grad, tau=tau, masked=masked)
    return dict(c, name=name) if name else c


def _verify(name, seqs, most, V, dtype, draft_probs, pad=0, sharp=4.0):
    c = dict(op="verify", seqs=seqs, most=most, V=V, pad=pad, dtype=dtype, draft_probs=draft_probs, sharp=sharp)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the candidates of one decoding step of four sequences: all latency
        _top("top_decode", 4, 10_000, 20, "float32"),
        # a teacher's lists for half a million tokens are written in pieces of this size
        _top("top_teacher", 4096, 131_072, 64, "bfloat16"),
        # long lists from an odd vocabulary with masked words, rows at odd addresses
        _top("top_odd_long", 777, 100_003, 301, "float16", pad=2, masked=True, tau=2.0),
        # a small drafter's step: a few rows, a small vocabulary
        _distill("distill_small", 16, 10_000, 16, "float32", True, True),
        # a drafter's training step, 2048 tokens, the vocabulary of the "large" corpus
        _distill("distill_train", 2048, 141_000, 64, "bfloat16", True, True, tau=2.0),
        # the same loss looked at without a gradient
        _distill("distill_eval", 4096, 100_000, 128, "float16", False, False),
        # odd sizes, padded rows and lists, masked words, in single precision
        _distill("distill_odd", 515, 50_021, 33, "float32", True, True, pad=2, masked=True, tau=1.5),
        # one sequence, four drafted tokens: all latency
        _verify("verify_one", 1, 4, 10_000, "float32", True),
        # a serving batch, ragged drafts
        _verify("verify_batch", 64, 7, 131_072, "float32", True),
        # a large batch on 16-bit probabilities
        _verify("verify_large", 256, 5, 141_000, "bfloat16", True),
        # drafts without probabilities (looked up in the text so far), the largest vocabulary
        _verify("verify_lookup", 33, 6, 1_000_000, "float32", False, pad=1, sharp=6.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["top", "distill", "verify"])
    dtype = rng.choice(list(DTYPES))
    V = _log_int(rng, 500, 1_000_000)
    pad = rng.choice([0, 0, 1, 2, 8, 13])
    if op == "verify":
        most = rng.randint(1, 8)
        seqs = _log_int(rng, 1, max(1, min(512, 200_000_000 // (V * (most + 1)))))
        return _verify(None, seqs, most, V, dtype, rng.random() < 0.7, pad, rng.choice([2.0, 4.0, 6.0]))
    rows = _log_int(rng, 1, max(1, min(8192, 280_000_000 // V)))
    top = _log_int(rng, 1, min(TOP_MOST, V))
    tau = rng.choice([0.7, 1.0, 1.0, 2.0, 4.0])
    masked = rng.random() < 0.4
    if op == "top":
        return _top(None, rows, V, top, dtype, pad, masked, tau)
    return _distill(None, rows, V, top, dtype, rng.random() < 0.6, rng.random() < 0.7, pad, masked, tau)


# --- inputs ------------------------------------------------------------------------------------------------------------------

def _padded(x, pad):
    """x with rows that lie `pad` values further apart than they are long."""
    if not pad:
        return x.contiguous()
    wide = x.new_zeros(x.shape[0], x.shape[1] + pad)
    wide[:, : x.shape[1]] = x
    return wide[:, : x.shape[1]]


def _logits(gen, rows, V, spread=2.0):
    """Logits as a model of text gives them: a bias that falls with the word's rank (words in no order), a normal part per
    place, and a few words that this place makes likely."""
    dev = "cuda"
    rank = torch.randperm(V, generator=gen, device=dev).float()
    x = torch.randn(rows, V, generator=gen, device=dev)
    x.mul_(spread).sub_(torch.log1p(rank))
    few = min(8, V)
    at = torch.randint(V, (rows, few), generator=gen, device=dev)
    x.scatter_add_(1, at, 6 + 4 * torch.rand(rows, few, generator=gen, device=dev))
    return x


def _masked_words(gen, V):
    """Words that may not be used: one in sixteen."""
    return torch.rand(V, generator=gen, device="cuda") < 1 / 16


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, V, dev = DTYPES[case["dtype"]], case["V"], "cuda"
    if case["op"] == "top":
        x = _logits(gen, case["rows"], V)
        if case["masked"]:
            x.masked_fill_(_masked_words(gen, V), -math.inf)
        return dict(case=case, logits=_padded(x.to(dt), case["pad"]))
    if case["op"] == "distill":
        rows, top, tau = case["rows"], case["top"], case["tau"]
        teacher = _logits(gen, rows, V)
        student = 0.8 * teacher
        student += torch.randn(rows, V, generator=gen, device=dev)
        weights = torch.full((rows,), (65536.0 if dt == torch.float16 else 1.0) / rows, device=dev)
        if case["masked"]:
            gone = _masked_words(gen, V)
            teacher.masked_fill_(gone, -math.inf)
            student.masked_fill_(gone, -math.inf)
        values, ids = torch.topk(teacher.to(dt).float(), top, dim=1)
        lse = torch.logsumexp(teacher.div_(tau), dim=1) if case["tail"] else None
        del teacher
        if case["masked"]:
            # lists of different lengths, and places of the batch that hold no token
            length = torch.randint(1, top + 1, (rows,), generator=gen, device=dev)
            length[torch.rand(rows, generator=gen, device=dev) < 1 / 8] = 0
            ids.masked_fill_(torch.arange(top, device=dev) >= length[:, None], -1)
            ids.masked_fill_(values == -math.inf, -1)
            weights.masked_fill_(length == 0, 0.0)
        return dict(case=case, logits=_padded(student.to(dt), case["pad"]), ids=ids.to(torch.int32),
                    values=values.to(dt), lse=lse, weights=weights)
    seqs, most = case["seqs"], case["most"]
    # ragged: every length up to the longest about equally often, in any order
    lengths = (most - torch.arange(seqs, device=dev) % (most + 1))[torch.randperm(seqs, generator=gen, device=dev)]
    offsets = torch.zeros(seqs + 1, dtype=torch.int64, device=dev)
    offsets[1:] = torch.cumsum(lengths, 0)
    n = int(offsets[-1])
    seq = torch.repeat_interleave(torch.arange(seqs, device=dev), lengths)
    x = _logits(gen, n + seqs, V)
    x.mul_(case["sharp"] / 4)
    target = _padded(torch.softmax(x, 1).to(dt), case["pad"])
    x = x[torch.arange(n, device=dev) + seq]
    x += 0.7 * torch.randn(n, V, generator=gen, device=dev)
    probs = torch.softmax(x, 1).to(dt)
    # the drafter's tokens: drawn from its probabilities
    cum = torch.cumsum(probs.float(), 1)
    u = torch.rand(n, 1, generator=gen, device=dev) * cum[:, -1:]
    drafts = (cum <= u).sum(1).clamp_(max=V - 1).to(torch.int32)
    return dict(case=case, offsets=offsets, drafts=drafts, target=target,
                probs=_padded(probs, case["pad"]) if case["draft_probs"] else None,
                accept_u=torch.rand(n, generator=gen, device=dev), draw_u=torch.rand(seqs, generator=gen, device=dev),
                tokens=torch.full((n + seqs,), -1, dtype=torch.int32, device=dev),
                accepted=torch.zeros(seqs, dtype=torch.int32, device=dev))


# --- the framework's calls ---------------------------------------------------------------------------------------------------

def _own(s):
    from paper_1412_1576_b200 import rows
    case = s["case"]
    if case["op"] == "top":
        ids, values, lse = rows.top_logits(s["logits"], case["top"], temperature=case["tau"])
        return dict(ids=ids, values=values, lse=lse)
    if case["op"] == "distill":
        if not case["grad"]:
            return dict(loss=rows.distill_loss(s["logits"], s["ids"], s["values"], s["lse"], temperature=case["tau"]))
        loss, grad = rows.distill_loss_and_grad(s["logits"], s["ids"], s["values"], s["lse"], temperature=case["tau"],
                                                weights=s["weights"])
        return dict(loss=loss, grad=grad)
    tokens, accepted = rows.verify_drafts(s["offsets"], s["drafts"], s["target"], s["probs"], s["accept_u"], s["draw_u"],
                                          tokens=s["tokens"], accepted=s["accepted"])
    return dict(tokens=tokens, accepted=accepted)


# --- the plain forms ---------------------------------------------------------------------------------------------------------

def _ordered(x):
    """Whole numbers in the order of the values (NaN above all, both zeros alike)."""
    b = (x + 0.0).view(torch.int32)
    return torch.where(torch.isnan(x), 0x7FFFFFFF, b ^ ((b >> 31) & 0x7FFFFFFF))


def _plain_top(case, logits):
    x = logits.float()
    V, dev = case["V"], x.device
    # value first, then the lower word: one whole number per word, all of them different
    key = _ordered(x).long() * 2**32 + (2**32 - 1 - torch.arange(V, device=dev))
    ids = torch.topk(key, case["top"], dim=1).indices
    del key
    values = torch.gather(logits, 1, ids)
    ids = ids.masked_fill(values == -math.inf, -1).to(torch.int32)
    x = x / case["tau"]
    m = x.max(1, keepdim=True).values
    lse = torch.log(torch.exp(x - m).sum(1)) + m[:, 0]
    return dict(ids=ids, values=values, lse=lse)


def _plain_distill(case, s):
    tau = case["tau"]
    x = s["logits"].float() / tau
    m = x.max(1, keepdim=True).values
    e = torch.exp(x - m)
    there = s["ids"] >= 0
    at = s["ids"].long().clamp(min=0)
    a = (s["values"].double() / tau).masked_fill(~there, -math.inf)
    # sums over the words of the list and over the others apart: neither is a difference of large sums
    listed_sum = torch.gather(e, 1, at).double().masked_fill(~there, 0.0).sum(1, keepdim=True)
    rest = e.scatter_add(1, at, torch.where(there, -torch.gather(e, 1, at), 0.0)).double().sum(1, keepdim=True)
    total = listed_sum + rest
    log_q = torch.gather(x, 1, at).double() - m - torch.log(total)
    if case["tail"]:
        log_p = a - s["lse"].double()[:, None]
        p = torch.exp(log_p)
        p_rest = (1 - p.sum(1, keepdim=True)).clamp(min=0)
    else:
        a_max = a.max(1, keepdim=True).values.clamp(min=-1e300)
        z = torch.exp(a - a_max).sum(1, keepdim=True)
        log_p = a - a_max - torch.log(z)
        p = torch.exp(log_p)
        p_rest = torch.zeros_like(total)
    empty = ~there.any(1, keepdim=True)
    p = p.masked_fill(empty | ~there, 0.0)
    p_rest = p_rest.masked_fill(empty | (rest == 0), 0.0)
    q_rest = rest / total
    loss = torch.where(p > 0, p * (log_p - log_q), 0.0).sum(1, keepdim=True)
    loss = loss + torch.where(p_rest > 0, p_rest * (torch.log(p_rest) - torch.log(q_rest)), 0.0)
    loss = (loss[:, 0] * tau * tau).float()
    if not case["grad"]:
        return dict(loss=loss)
    w = (s["weights"].double() * tau)[:, None]
    mass = p.sum(1, keepdim=True) + p_rest
    outside = torch.where(p_rest > 0, mass - p_rest / q_rest, mass)
    q_list = torch.gather(e, 1, at).double() / total
    g = e.mul_((w * outside / total).float())
    fix = torch.where(there, w * (q_list * (mass - outside) - p), 0.0)
    g.scatter_add_(1, at, fix.float())
    return dict(loss=loss, grad=g.to(s["logits"].dtype))


def _mass(r):
    return torch.floor(r.clamp(0.0, 1.0).double() * 2.0**MASS).long()


def _plain_verify(case, s):
    offsets, drafts, dev = s["offsets"], s["drafts"].long(), s["drafts"].device
    n, seqs = drafts.numel(), offsets.numel() - 1
    i = torch.arange(n, device=dev)
    seq = torch.searchsorted(offsets[1:], i, right=True)
    length = offsets[1:] - offsets[:-1]
    p = s["target"][i + seq, drafts].double()
    q = s["probs"][i, drafts].double() if s["probs"] is not None else torch.ones_like(p)
    taken = s["accept_u"].double() * q < p
    place = i - offsets[seq]
    accepted = length.scatter_reduce(0, seq, torch.where(taken, length[seq], place), "amin")
    row = offsets[:-1] + accepted
    refused = accepted < length
    p_row = s["target"][row + torch.arange(seqs, device=dev)].float()
    r = p_row
    if n:
        at = row.clamp(max=n - 1)
        if s["probs"] is not None:
            r = p_row - torch.where(refused[:, None], s["probs"][at].float(), 0.0)
        else:
            r = p_row.scatter(1, drafts[at][:, None], torch.where(refused[:, None], 0.0, p_row.gather(1, drafts[at][:, None])))
    mass = _mass(r)
    mass = torch.where(mass.sum(1, keepdim=True) > 0, mass, _mass(p_row))
    cum = torch.cumsum(mass, 1)
    total = cum[:, -1]
    u = torch.floor(s["draw_u"].double() * 2.0**32).long()
    # floor(total u / 2^32) in products of less than 2^63
    low = total & 0xFFFFFFFF
    x = (total >> 32) * u + ((low * (u >> 16) + ((low * (u & 0xFFFF)) >> 16)) >> 16)
    token = torch.where(total > 0, (cum <= x[:, None]).sum(1), -1).to(torch.int32)
    tokens = torch.full((n + seqs,), -1, dtype=torch.int32, device=dev)
    tokens[i + seq] = torch.where(place < accepted[seq], s["drafts"], -1)
    tokens[row + torch.arange(seqs, device=dev)] = token
    return dict(tokens=tokens, accepted=accepted.to(torch.int32))


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["op"] == "top":
        return _plain_top(case, state["logits"])
    return _plain_distill(case, state) if case["op"] == "distill" else _plain_verify(case, state)


def work(case):
    size, V = SIZES[case["dtype"]], case["V"]
    if case["op"] == "top":
        rows = case["rows"]
        return dict(bytes=rows * (V * size + case["top"] * (4 + size) + 4), flops=rows * V * 4)
    if case["op"] == "distill":
        rows = case["rows"]
        b = rows * (V * size * (2 if case["grad"] else 1) + case["top"] * (4 + size) + 8)
        return dict(bytes=b, flops=rows * V * (6 if case["grad"] else 4))
    # one row of the target per sequence, and one of the drafter where a draft is refused: in about half the sequences
    rows = case["seqs"] * (1 + (1 / 2 if case["draft_probs"] else 0))
    drafts = case["seqs"] * case["most"] / 2
    return dict(bytes=rows * V * size + drafts * (12 + 2 * size) + case["seqs"] * 24, flops=case["seqs"] * V * 3)


# --- the operators' definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_top(case, s):
    x = s["logits"].double()
    values, ids = torch.sort(x, dim=1, descending=True, stable=True)
    values, ids = values[:, : case["top"]].contiguous(), ids[:, : case["top"]].to(torch.int32)
    ids[values == -math.inf] = -1
    return dict(ids=ids, values=values.to(s["logits"].dtype), lse=torch.logsumexp(x / case["tau"], 1))


def _exact_distill(case, s):
    tau, rows, V = case["tau"], case["rows"], case["V"]
    loss = torch.zeros(rows, dtype=torch.float64, device="cuda")
    grad = torch.zeros(rows, V, dtype=torch.float64, device="cuda") if case["grad"] else None
    step = max(1, 100_000_000 // V)
    for lo in range(0, rows, step):
        hi = min(rows, lo + step)
        there = s["ids"][lo:hi] >= 0
        # one column more takes what is padding
        at = torch.where(there, s["ids"][lo:hi].long(), V)
        p = torch.full((hi - lo, V + 1), 0.0, dtype=torch.float64, device="cuda")
        t = (s["values"][lo:hi].double() / tau).masked_fill(~there, -math.inf)
        norm = s["lse"][lo:hi].double() if case["tail"] else torch.logsumexp(t, 1)
        p.scatter_add_(1, at, torch.nan_to_num(torch.exp(t - norm[:, None]), nan=0.0))
        p = p[:, :V]
        member = torch.zeros(hi - lo, V + 1, dtype=torch.bool, device="cuda").scatter_(1, at, True)[:, :V]
        log_q = torch.log_softmax(s["logits"][lo:hi].double() / tau, 1)
        out_q = torch.logsumexp(log_q.masked_fill(member, -math.inf), 1)
        out_p = (1 - p.sum(1)).clamp(min=0) if case["tail"] else torch.zeros_like(norm)
        out_p[(out_q == -math.inf) | ~there.any(1)] = 0.0
        terms = torch.where(p > 0, p * (torch.log(p) - log_q), 0.0).sum(1)
        loss[lo:hi] = tau * tau * (terms + torch.where(out_p > 0, out_p * (torch.log(out_p) - out_q), 0.0))
        if grad is not None:
            q = torch.exp(log_q)
            outside = torch.where(member, 0.0, torch.exp(log_q - out_q[:, None])) * out_p[:, None]
            outside[out_p == 0] = 0.0
            d = q * (p.sum(1) + out_p)[:, None] - p - outside
            grad[lo:hi] = d * (tau * s["weights"][lo:hi].double())[:, None]
    return dict(loss=loss) if grad is None else dict(loss=loss, grad=grad)


def _exact_verify(case, s):
    offsets, drafts = s["offsets"].tolist(), s["drafts"].tolist()
    u, d = s["accept_u"].tolist(), s["draw_u"].tolist()
    seqs, n = len(offsets) - 1, len(drafts)
    tokens, accepted = [-1] * (n + seqs), []
    for b in range(seqs):
        lo, hi = offsets[b], offsets[b + 1]
        i = lo
        while i < hi:
            q = float(s["probs"][i, drafts[i]]) if s["probs"] is not None else 1.0
            if not u[i] * q < float(s["target"][i + b, drafts[i]]):
                break
            tokens[i + b] = drafts[i]
            i += 1
        accepted.append(i - lo)
        p = s["target"][i + b].double()
        r = p.clone()
        if i < hi:
            if s["probs"] is not None:
                r = (p.float() - s["probs"][i].float()).double()
            else:
                r[drafts[i]] = 0.0
        for x in (r, p):
            mass = (x.clamp(0.0, 1.0) * 2.0**MASS).to(torch.int64)
            total = int(mass.sum())
            if total:
                want = total * int(d[b] * 2**32) >> 32
                tokens[i + b] = int(torch.searchsorted(torch.cumsum(mass, 0), want, right=True))
                break
    return dict(tokens=torch.tensor(tokens, dtype=torch.int32), accepted=torch.tensor(accepted, dtype=torch.int32))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "top":
        return _exact_top(case, s)
    return _exact_distill(case, s) if case["op"] == "distill" else _exact_verify(case, s)
