"""The operators of the training half that are measured: losses on logits with their gradients, and the global
gradient norm with clipping.

Four kinds of call:
  sar     Model.sar_loss_grad: the loss of semi-autoregressive finetuning and its gradient.
  policy  Model.policy_loss: clipped policy loss with a KL term, and its gradient.
  pref    Model.preference_loss: preference loss of paired log ratios, and its gradient.
  clip    Model.grad_clip: the norm over all gradients of a model (or some of its layers) and the clipped gradients.

Where `own` is false, run() computes the same in elementary torch operations.  Everything is drawn on the GPU from the
seed alone.  Logits are N(0, 2) with the label lifted on most rows, as a partly trained model's are.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"

# (layers, d_model, attention width, key/value width, ffn, vocabulary) of the repository's shapes whose gradients are clipped
_WIDTHS = {"tiny": (256, 256, 256, 688, 1000), "small128": (512, 512, 512, 1376, 2000), "gqa128": (1024, 1024, 512, 1376, 2000),
           "7b": (4096, 4096, 4096, 11008, 32000), "13b": (5120, 5120, 5120, 13824, 32000), "70b": (8192, 8192, 1024, 28672, 32000)}


# ------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # The loss on the logits of one decoding block (k = 5): the smallest call there is, launches and latencies.
        dict(name="sar_block_36", kind="sar", lens="36", prompt=0.0, pad=0, vocab=32000, dtype="f32", mean=False),
        # Two finetuning samples at the paper's caps (2048 tokens of prompt, 2048 of answer); the prompt does not count.
        dict(name="sar_8192_bf16", kind="sar", lens="4096,4096", prompt=0.5, pad=0, vocab=32000, dtype="bf16", mean=True),
        # A short sample over an odd vocabulary with 32-bit logits: rows at every alignment.
        dict(name="sar_333_odd", kind="sar", lens="333", prompt=0.3, pad=5, vocab=40001, dtype="f32", mean=True),
        # A single short rollout.
        dict(name="policy_61_bf16", kind="policy", lens="61", prompt=0.2, pad=0, vocab=32000, dtype="bf16", mean=True, kl=0.04, weighted=False, old=True),
        # Eight rollouts of one prompt, 32-bit logits, with a KL term towards a reference model.
        dict(name="policy_8x512_f32", kind="policy", lens="512,407,512,333,498,512,271,512", prompt=0.25, pad=0, vocab=32000, dtype="f32",
             mean=True, kl=0.04, weighted=True, old=True),
        # Many tokens of a small vocabulary.
        dict(name="policy_6001_v1000", kind="policy", lens="3000,3001", prompt=0.1, pad=0, vocab=1000, dtype="f32", mean=True, kl=0.0, weighted=False,
             old=True),
        # One pair of short answers.
        dict(name="pref_1x43_bf16", kind="pref", lens="24,19", prompt=0.2, pad=0, vocab=32000, dtype="bf16", mean=True, ref=True, average=False,
             smoothing=0.0),
        # A batch of eight pairs, ragged, prompts not counting, rows of padding behind the last.
        dict(name="pref_8_bf16", kind="pref", lens="512,433,301,390,777,512,256,299,512,501,640,333,128,190,460,512", prompt=0.4, pad=64, vocab=32000,
             dtype="bf16", mean=True, ref=True, average=False, smoothing=0.1),
        # The form without a reference model, mean log probabilities, odd vocabulary.
        dict(name="pref_2_odd_f32", kind="pref", lens="211,190,97,305", prompt=0.3, pad=0, vocab=5003, dtype="f32", mean=False, ref=False, average=True,
             smoothing=0.0),
        # A small model, gradients and result in 32 bits: launches and latencies.
        dict(name="clip_tiny_f32", kind="clip", shape="tiny", layers=2, heads=True, dtype="f32", out="f32", max_norm=1.0),
        # Layers of middling width, bf16 throughout, below the limit.
        dict(name="clip_gqa128_bf16", kind="clip", shape="gqa128", layers=12, heads=True, dtype="bf16", out="bf16", max_norm=1e6),
        # Two layers of the 7B shape with embedding and head: bf16 gradients into the optimiser's 32-bit ones.
        dict(name="clip_7b_2l_bf16", kind="clip", shape="7b", layers=2, heads=True, dtype="bf16", out="f32", max_norm=1.0),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["sar", "policy", "pref", "clip"])
    if kind == "clip":
        shape = rng.choice(["tiny", "small128", "gqa128", "7b", "13b", "70b"])
        most = {"tiny": 24, "small128": 24, "gqa128": 24, "7b": 2, "13b": 2, "70b": 1}[shape]
        heads = shape in ("tiny", "small128", "gqa128") or (shape == "7b" and rng.random() < 0.5)
        dtype = "bf16" if shape == "70b" or (heads and shape == "7b") else rng.choice(["f32", "bf16"])
        return dict(kind=kind, shape=shape, layers=rng.randint(1, most), heads=heads, dtype=dtype,
                    out=rng.choice(["f32", "bf16"]) if shape not in ("13b", "70b") else "bf16", max_norm=rng.choice([0.5, 1.0, 1e6]))
    vocab = rng.choice([1000, 2000, 32000, 32000, 32000, 5003, 40001, _log_int(rng, 1000, 64000)])
    dtype = rng.choice(["f32", "bf16"])
    rows = _log_int(rng, 8, max(9, min(8192, int(1.0e9 / (vocab * (8 if dtype == "f32" else 4))))))
    n_seq = 2 * rng.randint(1, 8) if kind == "pref" else rng.randint(1, 8)
    n_seq = max(2 if kind == "pref" else 1, min(n_seq, rows // 4 // 2 * 2))
    cut = sorted(rng.randint(0, rows) for _ in range(n_seq - 1))
    lens = ",".join(str(b - a) for a, b in zip([0] + cut, cut + [rows]))
    case = dict(kind=kind, lens=lens, prompt=rng.choice([0.0, 0.3, 0.5]), pad=rng.choice([0, 0, rng.randint(1, 40)]), vocab=vocab, dtype=dtype,
                mean=rng.random() < 0.7)
    if kind == "policy":
        case.update(kl=rng.choice([0.0, 0.04, 0.2]), weighted=rng.random() < 0.5, old=rng.random() < 0.8)
    if kind == "pref":
        case.update(ref=rng.random() < 0.7, average=rng.random() < 0.3, smoothing=rng.choice([0.0, 0.1]))
    return case


# -------------------------------------------------------------------------------------------- the inputs

CLIP_LOW, CLIP_HIGH, BETA, MARGIN = 0.2, 0.28, 0.1, 0.05


def _f32(v):
    """A parameter as the 32-bit number that a call gets."""
    return float(np.float32(v))


def _gen(seed, *where):
    words = np.random.SeedSequence([int(seed) & 0x7FFFFFFF, *where]).generate_state(2)
    return torch.Generator(device=DEV).manual_seed(int(words[0]) * (1 << 31) + int(words[1]) // 2)


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _logits_inputs(case, seed):
    lens, V = _lens(case), case["vocab"]
    rows = sum(lens) + case["pad"]
    g = _gen(seed, 1)
    x = torch.randn((rows, V), generator=g, device=DEV).mul_(2.0)
    labels = torch.randint(0, V, (rows,), generator=g, device=DEV, dtype=torch.int32)
    lift = torch.rand((rows, 1), generator=g, device=DEV) * 14.0
    x.scatter_add_(1, labels.long()[:, None], lift)
    x = x.to(_type(case["dtype"]))
    s = {"logits": x, "labels": labels, "rows": rows}
    if case["kind"] == "policy":
        # log probabilities of the model that made the rollouts and of the reference, near this one's
        logp = torch.empty(rows, device=DEV)
        for lo in range(0, rows, 1024):
            part = x[lo:lo + 1024].float()
            logp[lo:lo + 1024] = part.gather(1, labels[lo:lo + 1024].long()[:, None])[:, 0] - torch.logsumexp(part, 1)
        s["old_logp"] = logp + 0.2 * torch.randn(rows, generator=g, device=DEV) if case["old"] else None
        s["ref_logp"] = logp + 0.3 * torch.randn(rows, generator=g, device=DEV) if case["kl"] else None
        gain = torch.randn(len(lens), generator=g, device=DEV)
        n = torch.tensor(lens + [case["pad"]], device=DEV)
        s["advantages"] = torch.repeat_interleave(torch.cat([gain, gain.new_zeros(1)]), n, output_size=rows).contiguous()
        weight = torch.repeat_interleave(1.0 / n.clamp(min=1).float(), n, output_size=rows)
        s["row_weight"] = weight.contiguous() if case["weighted"] else None
    at = 0
    for n in lens:  # the prompt of every sequence does not count
        labels[at:at + int(n * case["prompt"])] = -1
        at += n
    labels[at:] = -1
    if case["kind"] == "pref":
        s["seq_start"] = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=DEV)
        if case["ref"]:
            per = 1.0 if case["average"] else torch.tensor([max(n, 1) for n in lens], device=DEV)
            s["ref_logp"] = -5.0 * per * (1 + 0.2 * torch.randn(len(lens), generator=g, device=DEV))
        else:
            s["ref_logp"] = None
    return s


def _tensor_shapes(case):
    d, hd, hkv, f, V = _WIDTHS[case["shape"]]
    one = [(d,), (hd, d), (hkv, d), (hkv, d), (d, hd), (d,), (f, d), (f, d), (d, f)]
    return case["layers"] * one + ([(V + 1, d), (d,), (V, d)] if case["heads"] else [])


def _grads(case, seed):
    shapes = _tensor_shapes(case)
    total = sum(math.prod(s) for s in shapes)
    spread = 3.0 / math.sqrt(total)  # a norm of a few units, tensors of unlike size
    return [torch.randn(s, generator=_gen(seed, 2, i), device=DEV).mul_(spread * (0.5 + (i * 7 % 5) / 4)).to(_type(case["dtype"]))
            for i, s in enumerate(shapes)]


def prepare(case, seed):
    if case["kind"] == "clip":
        grads = _grads(case, seed)
        flat = torch.empty(sum(g.numel() for g in grads), dtype=_type(case["out"]), device=DEV)  # what the optimiser reads
        outs, at = [], 0
        for g in grads:
            outs.append(flat[at:at + g.numel()].view(g.shape))
            at += g.numel()
        state = {"case": case, "grads": grads, "outs": outs, "flat": flat}
        if own:
            from paper_2402_11809_amd import binding
            model = _head_model(1000)
            state.update(model=model, set=binding.GradSet(model, grads, outs))
        return state
    state = dict(_logits_inputs(case, seed), case=case)
    if own:
        from paper_2402_11809_amd import binding
        model = _head_model(case["vocab"])
        pairs = len(_lens(case)) // 2 if case["kind"] == "pref" else 0
        # dlogits of sar and policy is the gradient of what is maximised, minus the loss: the calls are asked for it with a factor of -1
        state.update(model=model, out=binding.LossOut(model, state["rows"], grad_dtype=state["logits"].dtype, pairs=pairs),
                     minus=torch.full((1,), -1.0, device=DEV))
    return state


def _head_model(vocab):
    """A model of which only the vocabulary matters to these calls."""
    import gc
    from paper_2402_11809_amd import binding
    from space_inputs import ModelShape
    gc.collect()  # models that were dropped before; the library allocates beside torch
    shape = ModelShape("head-only", 1, 256, 4, 64, 688, vocab)
    zeros = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    return binding.Model(shape, {"embed": zeros(vocab + 1, 256), "lm_head": zeros(vocab, 256), "final_norm": zeros(256), "layers": [None]},
                         max_batch=1, max_rows=36, max_ctx=64)


# --------------------------------------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if own:
        return _run_own(case, s)
    return {"sar": _plain_sar, "policy": _plain_policy, "pref": _plain_pref, "clip": _plain_clip}[case["kind"]](case, s)


def _run_own(case, s):
    m = s["model"]
    if case["kind"] == "clip":
        return {"norm": m.grad_clip(s["set"], case["max_norm"]), "grads": s["flat"]}
    out = s["out"]
    if case["kind"] == "sar":
        m.sar_loss_grad(s["logits"], s["labels"], out, mean=case["mean"], grad_scale=s["minus"])
        return {"loss": out.loss, "n_terms": out.n_terms, "row_loss": out.row_loss, "dlogits": out.dlogits}
    if case["kind"] == "policy":
        m.policy_loss(s["logits"], s["labels"], s["advantages"], out, old_logp=s["old_logp"], ref_logp=s["ref_logp"], clip_low=CLIP_LOW,
                      clip_high=CLIP_HIGH, kl_coef=case["kl"], row_weight=s["row_weight"], mean=case["mean"], grad_scale=s["minus"])
        return {"loss": out.loss, "n_terms": out.n_terms, "row_loss": out.row_loss, "row_logp": out.row_logp, "n_clipped": out.n_clipped,
                "dlogits": out.dlogits}
    m.preference_loss(s["logits"], s["labels"], s["seq_start"], out, ref_logp=s["ref_logp"], beta=BETA, margin=MARGIN, smoothing=case["smoothing"],
                      average=case["average"], mean=case["mean"])
    return {"loss": out.loss, "pair_loss": out.pair_loss, "seq_logp": out.seq_logp, "row_logp": out.row_logp, "dlogits": out.dlogits}


def _plain_rows(s):
    """Exponentials below each row's maximum, their sum, the label's column and log probability, and which rows count."""
    x = s["logits"].float()
    keep = s["labels"] >= 0
    y = s["labels"].long().clamp(min=0)[:, None]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    logp = ((x.gather(1, y) - top).double() - torch.log(total))[:, 0]
    return e, total, y, torch.where(keep, logp, torch.zeros_like(logp)), keep


def _plain_gradient(s, e, total, y, c):
    """c[r] (onehot - softmax) of every row, c = dL / d log probability of the label."""
    c = c.float()[:, None]
    d = e * (-c / total.float())
    d.scatter_add_(1, y, c)
    return d.to(s["logits"].dtype)


def _plain_sar(case, s):
    e, total, y, logp, keep = _plain_rows(s)
    n = keep.sum()
    w = 1.0 / n.clamp(min=1) if case["mean"] else 1.0
    return {"loss": (-logp.sum() * w).float().view(1), "n_terms": n.int().view(1), "row_loss": -logp.float(),
            "dlogits": _plain_gradient(s, e, total, y, keep.double() * w)}


def _plain_policy(case, s):
    e, total, y, logp, keep = _plain_rows(s)
    n = keep.sum()
    old = s["old_logp"].double() if s["old_logp"] is not None else logp
    A = s["advantages"].double()
    q = torch.exp(logp - old)
    u, c = q * A, q.clamp(_f32(1 - _f32(CLIP_LOW)), _f32(1 + _f32(CLIP_HIGH))) * A
    clipped = keep & (u > c)
    term, g = -torch.minimum(u, c), torch.where(clipped, torch.zeros_like(u), u)
    if case["kl"]:
        d = s["ref_logp"].double() - logp
        term = term + _f32(case["kl"]) * (torch.expm1(d) - d)
        g = g + _f32(case["kl"]) * torch.expm1(d)
    if s["row_weight"] is not None:
        term, g = term * s["row_weight"].double(), g * s["row_weight"].double()
    w = 1.0 / n.clamp(min=1) if case["mean"] else 1.0
    term, g = torch.where(keep, term, torch.zeros_like(term)), torch.where(keep, g, torch.zeros_like(g))
    return {"loss": (term.sum() * w).float().view(1), "n_terms": n.int().view(1), "row_loss": term.float(), "row_logp": logp.float(),
            "n_clipped": clipped.sum().int().view(1), "dlogits": _plain_gradient(s, e, total, y, g * w)}


def _plain_pref(case, s):
    e, total, y, logp, keep = _plain_rows(s)
    S = s["seq_start"].numel() - 1
    row = torch.arange(s["rows"], device=DEV, dtype=torch.int32)
    seq = torch.bucketize(row, s["seq_start"][1:], right=True)  # S: behind the last sequence
    sums = torch.zeros(S + 1, dtype=torch.float64, device=DEV).index_add_(0, seq, logp)[:S]
    count = torch.zeros(S + 1, dtype=torch.float64, device=DEV).index_add_(0, seq, keep.double())[:S].clamp(min=1)
    if case["average"]:
        sums = sums / count
    ratio = sums if s["ref_logp"] is None else sums - s["ref_logp"].double()
    z = _f32(BETA) * (ratio[0::2] - ratio[1::2]) - _f32(MARGIN)
    eps = _f32(case["smoothing"])
    softplus = lambda v: v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))
    pair = (1 - eps) * softplus(-z) + eps * softplus(z)
    w = 1.0 / (S // 2) if case["mean"] else 1.0
    dz = (eps * torch.sigmoid(z) - (1 - eps) * torch.sigmoid(-z)) * (_f32(BETA) * w)
    per_seq = torch.stack([dz, -dz], 1).reshape(-1)
    if case["average"]:
        per_seq = per_seq / count
    c = torch.cat([per_seq, per_seq.new_zeros(1)])[seq] * keep
    return {"loss": (pair.sum() * w).float().view(1), "pair_loss": pair.float(), "seq_logp": sums.float(), "row_logp": logp.float(),
            "dlogits": _plain_gradient(s, e, total, y, c)}


def _plain_clip(case, s):
    square = sum((g.float() ** 2).sum(dtype=torch.float64) for g in s["grads"])
    norm = torch.sqrt(square)
    scale = torch.clamp(_f32(case["max_norm"]) / norm, max=1.0).float()
    for g, o in zip(s["grads"], s["outs"]):
        o.copy_(g.float() * scale)
    return {"norm": norm.float().view(1), "grads": s["flat"]}


# ------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "clip":
        n = sum(math.prod(s) for s in _tensor_shapes(case))
        size = {"f32": 4, "bf16": 2}
        return {"bytes": float(n * (size[case["dtype"]] + size[case["out"]])), "flops": 3.0 * n}
    lens, V, b = _lens(case), case["vocab"], 4 if case["dtype"] == "f32" else 2
    rows = sum(lens) + case["pad"]
    kept = sum(n - int(n * case["prompt"]) for n in lens)
    return {"bytes": float(b) * V * (kept + rows) + 16.0 * rows, "flops": 8.0 * kept * V}


# --------------------------------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    with torch.no_grad():
        return _exact_clip(case, seed) if case["kind"] == "clip" else _exact_loss(case, seed)


def _exact_clip(case, seed):
    grads = [g.double() for g in _grads(case, seed)]
    norm = math.sqrt(sum(float(torch.dot(g.flatten(), g.flatten())) for g in grads))
    limit = float(np.float32(case["max_norm"]))
    scale = limit / norm if norm > limit else 1.0
    return {"norm": torch.tensor([norm], dtype=torch.float64, device=DEV), "grads": torch.cat([g.flatten() for g in grads]) * scale}


def _exact_loss(case, seed):
    """Loss by loss from the log probabilities on the host; the gradient row by row as coefficient times (onehot - softmax)."""
    s = _logits_inputs(case, seed)
    rows, V = s["rows"], case["vocab"]
    labels = s["labels"].cpu().numpy()
    keep = labels >= 0
    logp = np.zeros(rows)
    for lo in range(0, rows, 512):
        x = s["logits"][lo:lo + 512].double()
        y = torch.from_numpy(np.maximum(labels[lo:lo + 512], 0).astype(np.int64)).to(DEV)
        logp[lo:lo + 512] = torch.log_softmax(x, 1).gather(1, y[:, None])[:, 0].cpu().numpy()
    logp[~keep] = 0.0
    coef, res = np.zeros(rows), {}
    if case["kind"] == "pref":
        start, pairs = s["seq_start"].cpu().numpy(), (s["seq_start"].numel() - 1) // 2
        ref = np.zeros(2 * pairs) if s["ref_logp"] is None else s["ref_logp"].double().cpu().numpy()
        beta, eps = float(np.float32(BETA)), float(np.float32(case["smoothing"]))
        total, weight = np.zeros(2 * pairs), 1.0 / pairs if case["mean"] else 1.0
        parts = [np.arange(start[i], start[i + 1])[keep[start[i]:start[i + 1]]] for i in range(2 * pairs)]
        for i, rs in enumerate(parts):
            total[i] = math.fsum(logp[rs]) / (max(len(rs), 1) if case["average"] else 1)
        loss = np.zeros(pairs)
        for p in range(pairs):
            z = beta * ((total[2 * p] - ref[2 * p]) - (total[2 * p + 1] - ref[2 * p + 1])) - float(np.float32(MARGIN))
            loss[p] = (1 - eps) * np.logaddexp(0.0, -z) + eps * np.logaddexp(0.0, z)
            slope = eps * np.exp(-np.logaddexp(0.0, -z)) - (1 - eps) * np.exp(-np.logaddexp(0.0, z))
            for which, sign in ((0, 1.0), (1, -1.0)):
                rs = parts[2 * p + which]
                coef[rs] = sign * beta * slope * weight / (max(len(rs), 1) if case["average"] else 1)
        res = {"loss": math.fsum(loss) * weight, "pair_loss": loss, "seq_logp": total, "row_logp": logp}
    elif case["kind"] == "sar":
        weight = 1.0 / max(int(keep.sum()), 1) if case["mean"] else 1.0
        coef[keep] = weight
        res = {"loss": -math.fsum(logp) * weight, "n_terms": None, "row_loss": -logp}
    else:
        weight = 1.0 / max(int(keep.sum()), 1) if case["mean"] else 1.0
        lo, hi = float(np.float32(1) - np.float32(CLIP_LOW)), float(np.float32(1) + np.float32(CLIP_HIGH))
        kl = float(np.float32(case["kl"]))
        adv = s["advantages"].double().cpu().numpy()
        old = logp if s["old_logp"] is None else s["old_logp"].double().cpu().numpy()
        ref = None if s["ref_logp"] is None else s["ref_logp"].double().cpu().numpy()
        scale = np.ones(rows) if s["row_weight"] is None else s["row_weight"].double().cpu().numpy()
        term = np.zeros(rows)
        for r in np.flatnonzero(keep):
            ratio = math.exp(logp[r] - old[r])
            inside = min(max(ratio, lo), hi)
            term[r] = max(-ratio * adv[r], -inside * adv[r])
            coef[r] = ratio * adv[r] if ratio * adv[r] <= inside * adv[r] else 0.0
            if kl:
                gap = ref[r] - logp[r]
                term[r] += kl * (math.expm1(gap) - gap)
                coef[r] += kl * math.expm1(gap)
        term, coef = term * scale, coef * scale * weight
        res = {"loss": math.fsum(term) * weight, "n_terms": None, "row_loss": term, "row_logp": logp, "n_clipped": None}
    grad = torch.empty(rows, V, dtype=torch.float64, device=DEV)
    for lo in range(0, rows, 512):
        x = s["logits"][lo:lo + 512].double()
        y = torch.from_numpy(np.maximum(labels[lo:lo + 512], 0).astype(np.int64)).to(DEV)
        one = torch.zeros_like(x).scatter_(1, y[:, None], 1.0)
        grad[lo:lo + 512] = torch.from_numpy(coef[lo:lo + 512]).to(DEV)[:, None] * (one - torch.softmax(x, 1))
    out = {k: None if v is None else torch.as_tensor(np.atleast_1d(v), dtype=torch.float64, device=DEV) for k, v in res.items()}
    out["dlogits"] = grad
    return out
