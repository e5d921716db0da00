"""What the tests of the losses on logits and of the gradient clipping share: a model of which only the vocabulary matters, the
formulas in 64 bits, and the tolerances.

Tolerances, with u = 2^-24 (half a step of a 32-bit number):
  * an exponential exp(x - top): x - top is rounded (|x - top| u on the exponent, so that much relative), the exponential itself
    is good to about an ulp (2 u, 4 u taken); a sum of them carries the same plus one u for each addition a thread makes in 32
    bits (fewer than 100): EXP = |x - top| + 4, SUM = EXP of the largest + 100, both in u, relative;
  * logp = (x_y - top) - log T: the first difference u of itself, the logarithm the sum's relative error, the result rounded once
    to 32 bits: (2 |logp| + SUM) u, absolute;
  * a gradient c e / T: the relative errors of c, e and T, two roundings; then the rounding to the logits' type
    (bf16: 2^-8, 32 bits: u).  What is below the smallest normal number may be flushed: 2 * 2^-126 absolute."""
import numpy as np

U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def head_model(V, max_rows=36):
    """A model without layers' weights: the losses read nothing but its vocabulary."""
    import torch
    from paper_2402_11809_amd import binding
    from space_inputs import ModelShape
    shape = ModelShape("head-only", 1, 32, 1, 64, 32, V)
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda:0")
    return binding.Model(shape, {"embed": z(V + 1, 32), "lm_head": z(V, 32), "final_norm": z(32), "layers": [None]},
                         max_batch=1, max_rows=max_rows, max_ctx=64)


def torch_type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def make_logits(rng, rows, V, dtype, std=2.0, lift=True):
    """(logits, labels): N(0, std), the label lifted on most rows, a fifth of the rows left out."""
    import torch
    x = (rng.standard_normal((rows, V)) * std).astype(np.float32)
    labels = rng.integers(0, V, size=rows).astype(np.int32)
    if lift:
        x[np.arange(rows), labels] += rng.uniform(0, 14, size=rows).astype(np.float32)
    if rows > 2:
        labels[rng.integers(0, rows, size=max(1, rows // 5))] = -1
    return torch.from_numpy(x).cuda().to(torch_type(dtype)), torch.from_numpy(labels).cuda()


class Rows64:
    """Rows of logits in 64 bits: logp of the label (0 where the row does not count), onehot - softmax, and the tolerances."""

    def __init__(self, logits, labels):
        import torch
        V = logits.shape[1]
        x = logits.double()
        self.keep = (labels >= 0) & (labels < V)
        y = labels.long().clamp(0, V - 1)[:, None]
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        T = e.sum(1, keepdim=True)
        logp = ((x.gather(1, y) - top) - torch.log(T))[:, 0]
        self.logp = torch.where(self.keep, logp, torch.zeros_like(logp))
        p = e / T
        others = e.scatter(1, y, 0.0).sum(1, keepdim=True)  # 1 - p of the label without a difference
        self.slope = (-p).scatter(1, y, others / T)         # onehot - softmax
        depth = torch.where(torch.isfinite(x), (top - x).clamp(min=0, max=104), torch.zeros_like(x))  # (deeper ones vanish)
        self.sum_tol = (depth.amax(1) + 104) * U            # relative error of T (and of others)
        self.elem_tol = (depth + 4) * U + self.sum_tol[:, None] + 4 * U
        self.logp_tol = (2 * self.logp.abs()) * U + self.sum_tol

    def check_logp(self, got, sign=1.0):
        import torch
        err = (got.double() * sign - self.logp).abs()
        assert bool((err <= self.logp_tol)[self.keep].all()), float((err / self.logp_tol)[self.keep].max())
        assert bool((got[~self.keep] == 0).all())

    def check_gradient(self, got, c, c_tol, dtype):
        """got against c (onehot - softmax), c = dL / d logp known to within c_tol (absolute)."""
        import torch
        c = torch.where(self.keep, c, torch.zeros_like(c))
        want = c[:, None] * self.slope
        tol = want.abs() * (self.elem_tol + HALF_STEP[dtype] * (1 + 2.0 ** -6)) + c_tol[:, None] * self.slope.abs() + 2.0 ** -125
        err = (got.double() - want).abs()
        rows = self.keep
        assert bool((err <= tol)[rows].all()), float((err / tol)[rows].max())
        assert bool((got[~rows] == 0).all()), "a row that does not count has a gradient"


def spoil(t):
    """Fills a tensor with what no correct result holds."""
    t.fill_(-7 if not t.is_floating_point() else float("nan"))
    return t


def fresh_out(gm, rows, dtype=None, **kw):
    from paper_2402_11809_amd import binding
    out = binding.LossOut(gm, rows, grad_dtype=None if dtype is None else torch_type(dtype), **kw)
    for n in ("loss", "n_terms", "row_logp", "row_loss", "row_kl", "n_clipped", "pair_loss", "seq_logp", "dlogits"):
        t = getattr(out, n)
        if t is not None and "dlogits" not in kw:
            spoil(t)
    spoil(out.work[4:])  # (an arrival count in front)
    return out
