"""The operators on arrays of logits whose speed is looked after: a teacher's top logits, the distillation criterion with
its gradient, and the verification of drafted words.

`listed()` holds the named cases, `draw()` gives further ones of the same ranges; `prepare()` builds what a program holds
before the call, `run()` is one call through the public binding (`own`) or the operator in elementary torch operations,
`work()` what one pass cannot do without, `exact()` the result from the definition in 64 bits.

A row of logits belongs to one window position: rows are time-major (position (t, s) is row t*B + s), and a row may be
longer than the vocabulary (`pad` more entries, as where a program keeps rows on 16-byte boundaries).
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # word prediction on a keyboard: the three likeliest next words of one text
        dict(name="top_wp10k_1", kind="top", rows=1, V=10000, pad=0, K=3, tau=1.0, dtype="bf16"),
        # a teacher reads a small window of a small corpus (vocabulary as counted, fp32)
        dict(name="top_odd_fp32", kind="top", rows=900, V=33278, pad=0, K=100, tau=2.0, dtype="fp32"),
        # a teacher of 64000 words over a whole training window of 128 streams
        dict(name="top_64k", kind="top", rows=2560, V=64000, pad=0, K=64, tau=1.0, dtype="bf16"),
        # a first experiment: toy vocabulary, a few streams, fp32
        dict(name="distill_toy_fp32", kind="distill", rows=32, V=1000, pad=0, K=8, tau=2.0, alpha=0.5, ragged=False,
             renorm=True, grad=True, dtype="fp32"),
        # a compressed word-prediction model taught by a large one, its teacher's distribution only
        dict(name="distill_wp10k", kind="distill", rows=2560, V=10000, pad=0, K=32, tau=2.0, alpha=1.0, ragged=False,
             renorm=False, grad=True, dtype="bf16"),
        # sizes nobody rounded, fp32; sentences of unequal length (positions without weight, labels missing, short lists)
        dict(name="distill_odd_fp32", kind="distill", rows=900, V=33278, pad=0, K=37, tau=1.5, alpha=0.7, ragged=True,
             renorm=True, grad=True, dtype="fp32"),
        # held-out loss of a student: no gradient
        dict(name="distill_eval_64k", kind="distill", rows=1280, V=64000, pad=0, K=64, tau=1.0, alpha=0.5, ragged=False,
             renorm=False, grad=False, dtype="bf16"),
        # the two large training windows: 128 streams of 20 words over 64000, 256 streams of 32 over 100000
        dict(name="distill_64k", kind="distill", rows=2560, V=64000, pad=0, K=64, tau=1.0, alpha=0.5, ragged=False,
             renorm=False, grad=True, dtype="bf16"),
        dict(name="distill_100k", kind="distill", rows=8192, V=100000, pad=0, K=100, tau=2.0, alpha=0.5, ragged=False,
             renorm=False, grad=True, dtype="bf16"),
        # one text, four drafted words
        dict(name="verify_wp10k_1", kind="verify", B=1, V=10000, pad=0, K=4, tau=1.0, filtered=False, ragged=False,
             drafter=True, dtype="bf16"),
        # texts side by side, drafts of unequal length from an n-gram that gives no probabilities; rare words masked
        dict(name="verify_odd_fp32", kind="verify", B=37, V=33278, pad=0, K=3, tau=0.8, filtered=True, ragged=True,
             drafter=False, dtype="fp32"),
        # a full batch against a small model's drafts
        dict(name="verify_100k", kind="verify", B=128, V=100000, pad=0, K=5, tau=1.0, filtered=False, ragged=True,
             drafter=True, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Vocabularies from 1000 to 131072 words (half of them round), from one row to the widest training window."""
    while True:
        V = _log_int(rng, 1000, 131072)
        if rng.random() < 0.5:
            V = max(1000, 250 * round(V / 250))
        case = dict(kind=rng.choice(["top", "distill", "distill", "verify"]), V=V, pad=rng.choice([0, 0, -V % 8, 24]),
                    dtype=rng.choice(["bf16", "bf16", "fp32"]), tau=rng.choice([1.0, 1.0, 2.0, 0.7, 3.5]))
        if case["kind"] == "top":
            case.update(rows=_log_int(rng, 1, 8192), K=_log_int(rng, 1, 256))
        elif case["kind"] == "distill":
            case.update(rows=_log_int(rng, 1, 8192), K=_log_int(rng, 1, 256), alpha=rng.choice([1.0, 0.5, 0.9]),
                        ragged=rng.random() < 0.4, renorm=rng.random() < 0.5, grad=rng.random() < 0.8)
        else:
            case.update(B=_log_int(rng, 1, 256), K=rng.randint(1, 8), filtered=rng.random() < 0.4,
                        ragged=rng.random() < 0.5, drafter=rng.random() < 0.7)
        if work(case)["bytes"] <= (work(listed()[8])["bytes"] if case["kind"] == "distill" else 1.2e9):
            return case


def _logits(gen, rows, V, pad, dtype, shared):
    """Rows of the logits a trained model gives: the words' overall frequency (Zipf) and what the context adds."""
    z = torch.empty(rows, V + pad, dtype=DTYPE[dtype], device="cuda")
    return z.normal_(0.0, 2.0, generator=gen)[:, :V].add_(shared)


def _zipf(gen, V):
    return torch.log(torch.randperm(V, generator=gen, device="cuda") + 10.0).neg_().add_(math.log(10.0))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    V, K, pad, dtype, kind = case["V"], case["K"], case["pad"], case["dtype"], case["kind"]
    shared = _zipf(gen, V)
    # scratch that a program keeps for such calls, whatever their sizes
    s = dict(case=case, workspace=torch.empty(256 << 20, dtype=torch.uint8, device="cuda"))
    if kind == "verify":
        B = case["B"]
        target = _logits(gen, (K + 1) * B, V, pad, dtype, shared)
        draft = target[: K * B].float().add_(torch.randn(K * B, V, generator=gen, device="cuda"), alpha=0.8).to(DTYPE[dtype])
        # drafts are drawn from the draft model's distribution (Gumbel's trick)
        e = torch.empty(K * B, V, device="cuda").exponential_(generator=gen)
        drafts = (draft.float() / case["tau"] - e.log_()).argmax(1)
        if case["filtered"]:  # words outside a shortlist are masked; the likeliest tenth of the words stays
            keep = shared >= shared.sort().values[int(0.9 * V)]
            target.masked_fill_(~keep, -math.inf)
        s["target"] = target.unflatten(0, (K + 1, B))
        s["draft"] = draft.unflatten(0, (K, B)) if case["drafter"] else None
        s["drafts"] = drafts.to(torch.int32).reshape(K, B)
        s["u"] = torch.rand(K + 1, B, generator=gen, device="cuda")
        s["lengths"] = torch.randint(0, K + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if case["ragged"] else None
        s["accepted"] = torch.empty(B, dtype=torch.int32, device="cuda")
        s["tokens"] = torch.empty(K + 1, B, dtype=torch.int32, device="cuda")
        return s
    M = case["rows"]
    s["logits"] = _logits(gen, M, V, pad, dtype, shared)
    s["ids"] = torch.empty(M, K, dtype=torch.int32, device="cuda")
    s["vals"] = torch.empty(M, K, device="cuda")
    s["lse"] = torch.empty(M, device="cuda")
    if kind == "top":
        return s
    # the teacher's list: distinct words, descending logits, and the logarithm of its whole sum
    first = torch.randint(0, V, (M, 1), generator=gen, device="cuda")
    step = 1 + torch.randint(0, max(1, V // K - 1), (M, 1), generator=gen, device="cuda")
    s["ids"].copy_((first + step * torch.arange(K, device="cuda")) % V)
    s["vals"].copy_((torch.randn(M, K, generator=gen, device="cuda") * 2.0).sort(1, descending=True).values)
    tail = torch.rand(M, generator=gen, device="cuda") * 0.3
    s["lse"].copy_(torch.logsumexp(s["vals"].double() / case["tau"], 1) - torch.log1p(-tail.double()))
    s["y"] = torch.randint(0, V, (M,), generator=gen, device="cuda", dtype=torch.int32)
    s["weight"] = None
    if case["ragged"]:
        s["weight"] = (torch.rand(M, generator=gen, device="cuda") < 0.8).float()
        s["y"][torch.rand(M, generator=gen, device="cuda") < 0.1] = -1
        s["ids"][torch.rand(M, K, generator=gen, device="cuda") < 0.2] = -1
    s["loss"] = torch.empty(M, device="cuda")
    s["dlogits"] = torch.empty(M, V + pad, dtype=DTYPE[dtype], device="cuda")[:, :V] if case["grad"] else None
    return s


def run(s):
    case = s["case"]
    tau, K, kind = case["tau"], case["K"], case["kind"]
    if own:
        from paper_1502_00512_amd import binding
        if kind == "top":
            ids, vals, lse = binding.rnnlm_top_logits(s["logits"], K, tau, s["ids"], s["vals"], s["lse"], s["workspace"])
            return dict(ids=ids, vals=vals, lse=lse)
        if kind == "distill":
            loss = binding.rnnlm_distill_loss(s["logits"], s["ids"], s["vals"], None if case["renorm"] else s["lse"],
                                              s["y"], s["weight"], tau, case["alpha"], 1.0 / case["rows"], s["loss"],
                                              s["dlogits"])
            return dict(loss=loss, dlogits=s["dlogits"]) if case["grad"] else dict(loss=loss)
        accepted, tokens = binding.rnnlm_verify_drafts(s["target"], s["drafts"], s["u"], s["draft"], s["lengths"], tau, tau,
                                                       s["accepted"], s["tokens"], s["workspace"])
        return dict(accepted=accepted, tokens=tokens)
    return {"top": _plain_top, "distill": _plain_distill, "verify": _plain_verify}[kind](s, case)


def _plain_top(s, case):
    z, tau = s["logits"].float(), case["tau"]
    # the greatest K of (value, lower id first): values as integers of the same order, the id below them
    bits = (z + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
    key = (order << 32) | (0x7FFFFFFF - torch.arange(case["V"], device=z.device))
    top = torch.topk(key, case["K"], dim=1).values
    ids = 0x7FFFFFFF - (top & 0x7FFFFFFF)
    m = z.max(1, keepdim=True).values
    lse = m / tau + torch.log(torch.exp((z - m) / tau).sum(1, keepdim=True))
    return dict(ids=ids.to(torch.int32), vals=z.gather(1, ids), lse=lse.squeeze(1))


def _plain_distill(s, case):
    z, tau, alpha = s["logits"].float(), case["tau"], case["alpha"]
    ids, there = s["ids"].long().clamp(min=0), s["ids"] >= 0
    t = (s["vals"] / tau).masked_fill(~there, -math.inf)
    norm = t.exp().sum(1, keepdim=True).log() if case["renorm"] else s["lse"][:, None]
    p = torch.where(there & torch.isfinite(t), (t - norm).exp(), 0.0)
    m = z.max(1, keepdim=True).values
    e = torch.exp((z - m) / tau)
    total = e.sum(1, keepdim=True)
    mass = p.sum(1, keepdim=True)
    ln_q = (z.gather(1, ids) - m) / tau - total.log()
    kd = torch.where(p > 0, p * (t - norm - ln_q), 0.0).sum(1)
    w = torch.ones_like(kd) if s["weight"] is None else s["weight"]
    y, has = s["y"].long().clamp(min=0)[:, None], s["y"] >= 0
    loss = alpha * tau * tau * kd
    if alpha < 1.0:
        e1 = e if tau == 1.0 else torch.exp(z - m)
        total1 = e1.sum(1, keepdim=True)
        hard = total1.log() - (z.gather(1, y) - m)
        loss = loss + (1.0 - alpha) * torch.where(has, hard.squeeze(1), 0.0)
    loss = w * loss
    if not case["grad"]:
        return dict(loss=loss)
    g = (w / case["rows"])[:, None]
    d = e * (alpha * tau * mass / total)
    if alpha < 1.0:
        d += e1 * ((1.0 - alpha) * has[:, None] / total1)
        d.scatter_add_(1, y, (alpha - 1.0) * has[:, None])
    d.scatter_add_(1, ids, -alpha * tau * p)
    return dict(loss=loss, dlogits=(d * g).to(s["logits"].dtype))


def _plain_verify(s, case):
    B, K, tau = case["B"], case["K"], case["tau"]

    def softmax(z):  # (in 64 bits: a word is chosen by which step of a long cumulated sum a number falls on)
        z = z.double() / tau
        e = torch.exp(z - z.max(2, keepdim=True).values)
        return e / e.sum(2, keepdim=True)

    p, at, d = softmax(s["target"]), torch.arange(B, device="cuda"), s["drafts"].long()[:, :, None]
    step = torch.arange(K, device="cuda")[:, None]
    q = softmax(s["draft"]) if s["draft"] is not None else None
    u = s["u"].double()
    length = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), K, device="cuda")
    ok = u[:K] * (1.0 if q is None else q.gather(2, d).squeeze(2)) < p[:K].gather(2, d).squeeze(2)
    n = (ok & (step < length)).long().cumprod(0).sum(0)
    last = n.clamp(max=K - 1)
    plain = p[n, at]
    taken = q[last, at] if q is not None else torch.zeros_like(plain).scatter_(1, d[last, at], 1.0)
    r = torch.where((n < length)[:, None], (plain - taken).clamp(min=0.0), plain)
    r = torch.where(r.sum(1, keepdim=True) > 0.0, r, plain)
    c = r.cumsum(1)
    word = (c <= u[K][:, None] * c[:, -1:]).sum(1)
    word = torch.minimum(word, torch.where(r > 0.0, torch.arange(case["V"], device="cuda"), -1).max(1).values)
    row = torch.arange(K + 1, device="cuda")[:, None]
    drafts = torch.cat([s["drafts"].long(), torch.zeros(1, B, dtype=torch.long, device="cuda")])
    tokens = torch.where(row < n, drafts, torch.where(row == n, word, -1))
    return dict(accepted=n.to(torch.int32), tokens=tokens.to(torch.int32))


def work(case):
    es, V, K = (4 if case["dtype"] == "fp32" else 2), case["V"], case["K"]
    if case["kind"] == "top":
        M = case["rows"]
        return {"bytes": M * (es * V + 8 * K + 4), "flops": 3.0 * M * V}
    if case["kind"] == "distill":
        M, temps = case["rows"], 2 if case["alpha"] < 1.0 and case["tau"] != 1.0 else 1
        return {"bytes": M * (es * V * (2 if case["grad"] else 1) + 8 * K + 12),
                "flops": 3.0 * M * V * temps * (2 if case["grad"] else 1)}
    B, rows = case["B"], (2 * K + 1 if case["drafter"] else K + 1) * case["B"]
    return {"bytes": rows * es * V + 4 * B * (3 * K + 4), "flops": 3.0 * rows * V}


def exact(case, seed):
    """From the definitions, block of rows by block of rows."""
    s, kind, tau = prepare(case, seed), case["kind"], case["tau"]
    if kind == "verify":
        return None  # whole numbers only
    M, z = case["rows"], s["logits"]
    block = max(1, int(2.5e8) // case["V"])
    parts = []
    for a in range(0, M, block):
        x = z[a: a + block].to(torch.float64)
        ln_q = torch.log_softmax(x / tau, 1)
        if kind == "top":
            parts.append(dict(ids=None, vals=x.topk(case["K"], 1).values, lse=torch.logsumexp(x / tau, 1)))
            continue
        ids = s["ids"][a: a + block].long()
        t = torch.where(ids >= 0, s["vals"][a: a + block].double() / tau, -math.inf)
        p = torch.exp(t - torch.logsumexp(t, 1, keepdim=True)) if case["renorm"] else torch.exp(t - s["lse"][a: a + block, None].double())
        p = torch.nan_to_num(p, nan=0.0)
        ln_p = torch.where(p > 0, torch.log(p), 0.0)
        teacher = torch.zeros_like(x).scatter_add_(1, ids.clamp(min=0), p)
        w = torch.ones(len(x), dtype=torch.float64, device="cuda") if s["weight"] is None else s["weight"][a: a + block].double()
        y = s["y"][a: a + block].long()
        label = torch.zeros_like(x).scatter_(1, y.clamp(min=0)[:, None], (y >= 0).double()[:, None])
        ln_1 = torch.log_softmax(x, 1)
        kd = (p * ln_p).sum(1) - (teacher * ln_q).sum(1)
        alpha = case["alpha"]
        part = dict(loss=w * (alpha * tau ** 2 * kd - (1 - alpha) * (label * ln_1).sum(1)))
        if case["grad"]:
            d = alpha * tau * (teacher.sum(1, keepdim=True) * ln_q.exp() - teacher)
            d += (1 - alpha) * (label.sum(1, keepdim=True) * ln_1.exp() - label)
            part["dlogits"] = d * w[:, None] / M
        parts.append(part)
    return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}
