"""The prompt-side operators in 64 bits, from their formulas, and the tolerances that their arithmetic allows."""
import math

import torch

D = 128
NEG = float("-inf")


def rope64(x, weight, eps, positions, inv_freq, interleaved):
    """x [n, heads, D], positions [n] -> rotated rows in 64 bits, and the size |a| + |b| of what each channel is summed from."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    size = y.abs()
    if inv_freq is None:
        return y, size
    half = inv_freq.numel()
    f = positions.double()[:, None] * inv_freq.double()
    c, s = torch.cos(f)[:, None], torch.sin(f)[:, None]
    i = torch.arange(half, device=x.device)
    lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = y[..., lo], y[..., hi]
    out = y.clone()
    out[..., lo], out[..., hi] = a * c - b * s, a * s + b * c
    size[..., lo] = size[..., hi] = a.abs() + b.abs()
    return out, size


def rope_tolerance(ref, size, dtype):
    # binary32: the mean of 128 squares (8 sums and 4 levels, so at most 13 roundings, half of which the root passes on),
    # root, quotient, product with the weight, sine or cosine to 2 units, two products and a sum: below 24 half units; then
    # one rounding to 16 bits, below fp16's normal range by half of its smallest step
    return ref.abs() * torch.finfo(dtype).eps / 2 * (1 + 2 ** -10) + size * 24 * 2 ** -24 + 2 ** -25


def gather_cache(cache, table, b, length):
    """Rows [Hkv, length, D] of a sequence and whether each token has a page."""
    if table is None:
        return cache[b, :, :length], torch.ones(length, dtype=torch.bool, device=cache.device)
    page = cache.shape[2]
    j = torch.arange(length, device=cache.device)
    at = table[b].long()[j // page]
    there = (at >= 0) & (at < cache.shape[0])
    rows = cache[at.clamp(0, cache.shape[0] - 1), :, j % page].transpose(0, 1).clone()
    rows[:, ~there] = 0
    return rows, there


def attn64(q, k, v, there, past, scale):
    """q [n, Hq, D], k and v [Hkv, L, D] -> out, lse, and the pieces that the tolerances need."""
    n, Hq, _ = q.shape
    Hkv, L, _ = k.shape
    R = Hq // Hkv
    qd = q.double().unflatten(1, (Hkv, R)).permute(1, 2, 0, 3).reshape(Hkv, R * n, D)
    kd = k.double()
    z = torch.matmul(qd, kd.transpose(1, 2).contiguous()).view(Hkv, R, n, L) * scale
    size = torch.matmul(qd.abs(), kd.abs().transpose(1, 2).contiguous()).view(Hkv, R, n, L) * scale
    ok = (torch.arange(L, device=q.device)[None] <= past + torch.arange(n, device=q.device)[:, None]) & there[None]
    z = z.masked_fill(~ok, NEG)
    m = z.amax(-1, keepdim=True)
    p = torch.where(ok, torch.exp(z - torch.where(m == NEG, 0.0, m)), 0.0)
    l = p.sum(-1, keepdim=True)
    w = p / torch.where(l > 0, l, 1.0)
    lse = (m + l.log())[..., 0]  # -inf where a row is empty
    out = spread = None
    if v is not None:
        out = torch.matmul(w.view(Hkv, R * n, L), v.double()).view(Hkv, R, n, D)
        spread = torch.matmul(w.view(Hkv, R * n, L), v.double().abs()).view(Hkv, R, n, D)
        out, spread = (x.permute(2, 0, 1, 3).reshape(n, Hq, D) for x in (out, spread))
    # a logit: 128 products and their sums in binary32 (2^-23 a step: the matrix units may truncate), scale and exponent
    dz = (132 * 2 ** -23 * torch.where(ok, size, 0.0)).amax(-1)
    rows = lambda x: x.permute(2, 0, 1).reshape(n, Hq)
    return dict(out=out, spread=spread, lse=rows(lse), dz=rows(dz), z=z, ok=ok, size=size, L=L)


def out_tolerance(r, dtype, out_dtype, vmax):
    """Weights carry the logits' errors (to and fro: twice), their sums one rounding a token.  16-bit outputs: a weight is
    rounded to 16 bits once, the result once more.  binary32 outputs: a weight keeps its rest as a second 16-bit number.
    fp16 weights lose what lies below half their smallest step, 2^-25 of the row's largest."""
    eps = torch.finfo(dtype).eps
    half = eps / 2 if out_dtype != torch.float32 else eps * eps / 4
    rel = half + 2 * r["dz"][..., None] + (r["L"] + 16) * 2 ** -23
    tol = r["spread"] * rel + r["out"].abs() * 2 ** -22
    if dtype == torch.float16:
        tol = tol + r["L"] * 2 ** -25 * vmax
    if out_dtype != torch.float32:
        tol = tol + r["out"].abs() * eps / 2 * (1 + 2 ** -8) + tol * eps + 2 ** -25
    return tol + 1e-30


def lse_tolerance(r):
    return r["dz"] + r["lse"].abs() * 2 ** -22 + (r["L"] + 16) * 2 ** -23


def mass64(r, lse, n_obs):
    """Weights received [Hkv, L] from the last n_obs of the n query rows of r against the given lse [n, Hq], and how far a
    binary32 evaluation may be off."""
    Hkv, R, n, L = r["z"].shape
    l = lse.double().view(n, Hkv, R).permute(1, 2, 0)[..., None]
    use = r["ok"] & (l > NEG)
    use = use & (torch.arange(n, device=lse.device) >= n - n_obs)[None, None, :, None]
    p = torch.where(use, torch.exp(r["z"] - torch.where(l > NEG, l, 0.0)), 0.0)
    # relative error of a weight: its logit (as above, and four half units of logit and lse each for scaling and base),
    # the exponential; of the sum: one rounding for each of the rows
    e = 132 * 2 ** -23 * r["size"] + 2 ** -21 * (torch.where(use, r["z"], 0.0).abs() + torch.where(l > NEG, l, 0.0).abs()) + 2 ** -22
    total = p.sum((1, 2))
    return total, (p * e).sum((1, 2)) + total * (n * R + 4) * 2 ** -24


def keep64(mass, length, n_keep, n_sink, n_recent):
    """Indices that stay, ascending, from a stable sort."""
    if length <= n_keep:
        return list(range(length))
    m = mass.tolist()
    middle = sorted(range(n_sink, length - n_recent), key=lambda i: -m[i])[:n_keep - n_sink - n_recent]
    return [*range(n_sink), *sorted(middle), *range(length - n_recent, length)]


SCALE = 1.0 / math.sqrt(D)


def out_tolerance_by_tile(r, v, dtype, out_dtype):
    """As out_tolerance, but for what fp16 weights lose: not 2^-25 of the row's largest for each token, but of the largest of
    the token's own 64, which is held at 2^-5 or more (binary32 results: 2^-1), and 2^-90 of the row's where a tile lies too deep
    for that.  v [Hkv, L, D]."""
    Hkv, R, n, L = r["z"].shape
    w = torch.exp(r["z"] - torch.logsumexp(r["z"], -1, keepdim=True)).nan_to_num(0.0)
    lost = torch.zeros_like(w)
    if dtype == torch.float16:
        top = torch.nn.functional.pad(w, (0, -L % 64)).unflatten(-1, (-1, 64)).amax(-1, keepdim=True).expand(-1, -1, -1, -1, 64)
        lost = top.flatten(-2)[..., :L] * (2 ** -24 if out_dtype == torch.float32 else 2 ** -20) + 2 ** -90
        lost = torch.where(r["ok"], lost, 0.0)
    eps = torch.finfo(dtype).eps
    half = eps / 2 if out_dtype != torch.float32 else eps * eps / 4
    rel = (half + 2 * r["dz"][..., None] + (r["L"] + 16) * 2 ** -23)
    lost = torch.matmul(lost.view(Hkv, R * n, L), v.double().abs()).view(Hkv, R, n, D).permute(2, 0, 1, 3).reshape(n, Hkv * R, D)
    tol = r["spread"] * rel + lost + r["out"].abs() * 2 ** -22
    if out_dtype != torch.float32:
        tol = tol + r["out"].abs() * eps / 2 * (1 + 2 ** -8) + tol * eps + (2 ** -25 if dtype == torch.float16 else 0.0)
    return tol + 1e-37
