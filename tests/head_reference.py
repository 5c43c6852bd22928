"""Norm, token log probabilities and distillation from their definitions in 64 bits (torch, any device), sharing no code with
the library.  Lists of the distillation are walked in Python."""
import math

import torch

HALF = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16, torch.float32)}   # a rounding, as a share of the value
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half the smallest subnormal


def norm(x, weight=None, bias_vec=None, residual=None, eps=1e-5, layer=True):
    """(h, y, mean, rstd); h in x's type (the statistics are of the stored sum), the others in 64 bits."""
    h = x if residual is None else (x.double() + residual.double()).to(x.dtype)
    y, mean, rstd = norm_of(h.double(), weight, bias_vec, eps, layer)
    return h, y, mean, rstd


def norm_of(h, weight, bias_vec, eps, layer):
    mean = h.mean(-1) if layer else torch.zeros_like(h[:, 0])
    dev = h - mean.unsqueeze(-1)
    rstd = 1.0 / torch.sqrt((dev * dev).mean(-1) + eps)
    y = dev * rstd.unsqueeze(-1)
    if weight is not None:
        y = y * weight.double()
    return y if bias_vec is None else y + bias_vec.double(), mean, rstd


def norm_grad(dy, h, weight, dh=None, eps=1e-5, layer=True):
    """(dx, dw, db) in 64 bits."""
    h, dy = h.double(), dy.double()
    _, mean, rstd = norm_of(h, None, None, eps, layer)
    rstd = rstd.unsqueeze(-1)
    xh = (h - mean.unsqueeze(-1)) * rstd
    g = dy if weight is None else dy * weight.double()
    dx = g - xh * (g * xh).mean(-1, keepdim=True)
    if layer:
        dx = dx - g.mean(-1, keepdim=True)
    dx = dx * rstd
    return (dx if dh is None else dx + dh.double()), (dy * xh).sum(0), dy.sum(0)


def log_softmax(logits, scale):
    """(log probabilities, ln of the sum) in 64 bits; rows of -infinity stay -infinity.  The largest goes first: a mask of
    -3e38 and a logarithm have no sum in 64 bits."""
    x = logits.double()
    most = x.amax(-1, keepdim=True)
    none = most == -math.inf
    z = scale * torch.where(none, x, x - most)
    logsum = torch.logsumexp(z, -1, keepdim=True)
    return torch.where(none, x, z - logsum), torch.where(none, most, scale * most + logsum).squeeze(-1)


def entropy(lp):
    return -torch.where(lp > -math.inf, lp.exp() * lp, torch.zeros_like(lp)).sum(-1)


def top(logits, k):
    """Indices by falling logit, equal ones by rising index (-0 equals 0)."""
    return torch.sort(logits.double() + 0.0, dim=-1, descending=True, stable=True).indices[:, :k]


def token_grad(logits, targets, g_logprob, g_entropy, scale):
    lp, _ = log_softmax(logits, scale)
    p = lp.exp()
    n, vocab = lp.shape
    out = torch.zeros_like(lp)
    if g_logprob is not None:
        given = (targets >= 0) & (targets < vocab)
        g = torch.where(given, g_logprob.double(), torch.zeros_like(p[:, 0]))
        row = torch.arange(n, device=lp.device)
        out = -g.unsqueeze(1) * p
        out[row[given], targets[given].long()] += g[given]
    if g_entropy is not None:
        h = entropy(lp).unsqueeze(1)
        out = out - g_entropy.double().unsqueeze(1) * torch.where(p > 0, p * (lp + h), torch.zeros_like(p))
    out = torch.where((lp == -math.inf).all(-1, keepdim=True), torch.zeros_like(out), out)
    return scale * out


def teacher_of(index, value, vocab, rest):
    """Of one row: {token: (q, ln q)} and the q of the rest."""
    entries = {}
    for j, v in zip(index, value):
        if 0 <= j < vocab and j not in entries:
            entries[j] = v
    if not entries:
        return {}, 0.0
    if not rest:
        most = max(entries.values())
        if most == -math.inf:
            return {}, 0.0
        lse = most + math.log(sum(math.exp(v - most) for v in entries.values()))
        return {j: (math.exp(v - lse), v - lse) for j, v in entries.items()}, 0.0
    total = sum(math.exp(v) for v in entries.values())
    return {j: (math.exp(v), v) for j, v in entries.items()}, max(0.0, 1.0 - total)


def distill(logits, index, value, rest, scale):
    """(loss [rows], gradient of each row's loss [rows, vocab]) in 64 bits."""
    lp, _ = log_softmax(logits, scale)
    rows, vocab = lp.shape
    loss, grad = [], torch.zeros_like(lp)
    for r in range(rows):
        q, left = teacher_of(index[r].tolist(), value[r].tolist(), vocab, rest)
        at = torch.tensor(sorted(q), dtype=torch.long, device=lp.device)
        qs = torch.tensor([q[j][0] for j in sorted(q)], dtype=torch.float64, device=lp.device)
        lq = torch.tensor([q[j][1] for j in sorted(q)], dtype=torch.float64, device=lp.device)
        p = lp[r].exp()
        unlisted = lp[r].clone()
        unlisted[at] = -math.inf
        if bool((unlisted == -math.inf).all()):
            left = 0.0                                    # no other token can come
        mass = float(qs.sum()) + left
        if mass == 0.0:
            loss.append(0.0)
            continue
        if bool((p == 0).all()):
            loss.append(math.inf)
            continue
        total = float(torch.where(qs > 0, qs * (lq - lp[r, at]), torch.zeros_like(qs)).sum())
        g = mass * p
        if left > 0.0:
            others = p.clone()
            others[at] = 0.0
            p_left = float(others.sum())
            total += left * (math.log(left) - math.log(p_left))
            g = g - others * (left / p_left)
        g[at] -= qs
        loss.append(total)
        grad[r] = scale * g
    return torch.tensor(loss, dtype=torch.float64, device=lp.device), grad
