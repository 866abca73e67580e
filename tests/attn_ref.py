"""Attention in 64 bits for the window and decode tests, and how far a result in 16 bits may be from it."""
import torch

BF16, FP32 = 2.0 ** -8, 2.0 ** -24          # half a step of the type, relative


def attend(q, k, v, pos, window=0, n_sink=0, scale=None, k_size=None, v_size=None, v_sum=None):
    """q [rows][H_q][D] at positions pos [rows], k / v [T][H_kv][D] -> out, lse, and what the bounds below need:
    sum of p |v| of every output and the largest sum of |q_i k_i| scale of every row (k_size, v_size: the sizes of the terms that
    the products are summed from, where those are not k and v; v_sum: of what the value products' sums pass through)."""
    q, k, v = q.double(), k.double(), v.double()
    g = q.shape[1] // k.shape[1]
    scale = q.shape[2] ** -0.5 if scale is None else scale
    kk, vv = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    key, p = torch.arange(k.shape[0], device=q.device), pos[:, None]
    seen = key <= p
    if window:
        seen &= (key < n_sink) | (key > p - window)
    seen = seen[:, None]
    bad = ~seen.any(0).any(0)                # keys nobody sees count as if they were not there, whatever they hold
    kk, vv = kk.masked_fill(bad[:, None, None], 0.0), vv.masked_fill(bad[:, None, None], 0.0)
    s = (torch.einsum("rhd,thd->rht", q, kk) * scale).masked_fill(~seen, -torch.inf)
    ka = kk.abs() if k_size is None else k_size.double().repeat_interleave(g, 1)
    va = vv.abs() if v_size is None else v_size.double().repeat_interleave(g, 1)
    size = (torch.einsum("rhd,thd->rht", q.abs(), ka) * abs(scale)).masked_fill(~seen, 0.0).amax(-1)
    lse = torch.logsumexp(s, -1)
    w = torch.exp(s - lse[..., None])
    vs = va if v_sum is None else v_sum.double().repeat_interleave(g, 1)
    return torch.einsum("rht,thd->rhd", w, vv), lse, torch.einsum("rht,thd->rhd", w, va), size, torch.einsum("rht,thd->rhd", w, vs)


def check(out, lse, want, keys, what=""):
    """Weights and results are rounded to bf16 once each; scores are sums of D products in fp32 (each at most a step off),
    whose error reaches the weights and the log-sum-exp as a factor; the sums of weights and of values run over `keys` terms, each
    up to a step of the sum off (4-bit values: c and -8 of a code enter one after the other)."""
    o, l, size_v, size_s, size_sum = want
    score = out.shape[-1] * 2 * FP32 * size_s + 4 * FP32 * size_s + 2.0 ** -21
    tol = BF16 * (size_v + o.abs()) * 1.01 + 2 * score[..., None] * size_sum + (keys + 16) * 2 * FP32 * size_sum + 1e-30
    assert torch.equal(out.isfinite(), o.isfinite()), what + ": not finite"
    err = (out.double() - o).abs() / tol
    err = err[o.isfinite()]
    worst = err.max().item() if err.numel() else 0.0
    assert worst <= 1.0, "%s: out %.3g times its bound" % (what, worst)
    if lse is not None:
        ltol = score + keys * FP32 + 4 * FP32 * l.abs() + 2.0 ** -20
        assert torch.equal(lse.isfinite(), l.isfinite()), what + ": lse not finite"
        lerr = ((lse.double() - l).abs() / ltol)[l.isfinite()]
        lworst = lerr.max().item() if lerr.numel() else 0.0
        assert lworst <= 1.0, "%s: lse %.3g times its bound" % (what, lworst)
