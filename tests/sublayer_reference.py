"""The attention sublayer's operators in 64 bits on the CPU, as their definitions read, with gradients by differentiation; and how far a result may be off.

Bounds, from the arithmetic alone.  bf16: a value is rounded by at most 2^-8 of itself; a result is rounded once, what it was summed from (probabilities, their gradients, the
outputs in do . o) at most twice more, each by an independent rounding of every term: over a whole tensor at most 3 x 2^-8 / sqrt(3) of its norm, taken as 2^-7.  A single entry may be the
small difference of terms as large as the tensor's largest: 2^-6 of that.  fp32: the same with 2^-24, times 64 for sums of up to some thousand terms and for exponentials whose arguments, up to
2^6, are rounded to 2^-24 of themselves.
What goes through ds = p (dp - do . o) is a difference that may cancel altogether: a row that sees one key, and a table of one bucket, have a gradient of exactly zero.  Its terms' roundings
stay: 2^-9 of the terms p (|dp| + |do . o|) in bf16, where o comes rounded by as much on average, 8 x 2^-24 in fp32, summed as the result is."""
import math

import torch

NORM = {torch.bfloat16: 2.0 ** -7, torch.float32: 64 * 2.0 ** -24}
MOST = {torch.bfloat16: 2.0 ** -6, torch.float32: 256 * 2.0 ** -24}


TERMS = {torch.bfloat16: 2.0 ** -9, torch.float32: 8 * 2.0 ** -24}


def check(got, want, name, as_type=None, terms=None):
    """Against the bounds of its type; infinities and NaN have to be where they are.  terms: the same sum with the absolute values of what may cancel."""
    t = as_type or got.dtype
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), f"{name}: finite in other places"
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[torch.isinf(want)], want[torch.isinf(want)]), name
    if not fine.any():
        return
    d, w = (got - want)[fine], want[fine]
    more = torch.zeros_like(w) if terms is None else TERMS[t] * terms.double().cpu()[fine]
    bound, most = NORM[t] * float(w.norm()) + float(more.norm()), MOST[t] * float(w.abs().max()) + float(more.max())
    assert float(d.norm()) <= bound and float(d.abs().max()) <= most, f"{name}: off by {float(d.norm()):.3g} (bound {bound:.3g}, norm {float(w.norm()):.3g}), at most {float(d.abs().max()):.3g} (bound {most:.3g})"


def attention(q, k, v, bias=None, bias_map=None, causal=False, scale=None, q_lengths=None, k_lengths=None, q_start=None, dout=None):
    """out, lse (and dq, dk, dv, dbias and the terms of dq, dk and dbias where dout is given) in 64 bits.  Hidden keys and rows are left out, not multiplied by zero."""
    b, n_q, heads, dim = q.shape
    n_k, group = k.shape[1], heads // k.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    leaves = [None if t is None else t.detach().cpu().double().requires_grad_(True) for t in (q, k, v, bias)]
    q, k, v, bias = leaves
    m = None if bias_map is None else bias_map.cpu().long()
    reach = 0 if m is None else m.numel() // 2
    out, lse = torch.zeros(b, n_q, heads, dim, dtype=torch.float64), torch.full((b, heads, n_q), -math.inf, dtype=torch.float64)
    total = torch.zeros((), dtype=torch.float64)
    terms = dict(dq=torch.zeros_like(q.detach()), dk=torch.zeros_like(k.detach()), dbias=None if bias is None else torch.zeros_like(bias.detach()))
    for n in range(b):
        rows = n_q if q_lengths is None else max(0, min(n_q, int(q_lengths[n])))
        cols = n_k if k_lengths is None else max(0, min(n_k, int(k_lengths[n])))
        first = 0 if q_start is None else int(q_start[n])
        for i in range(rows):
            seen = min(cols, first + i + 1) if causal else cols
            if seen <= 0:
                continue
            x = torch.einsum("hgd,jhd->hgj", q[n, i].view(-1, group, dim), k[n, :seen]).reshape(heads, seen) * scale
            if bias is not None:
                x = x + bias[m[(torch.arange(seen) - (first + i)).clamp(-reach, reach) + reach]].t()
            row_lse = torch.logsumexp(x, -1)
            p = torch.exp(x - row_lse[:, None])
            row = torch.einsum("hgj,jhd->hgd", p.view(-1, group, seen), v[n, :seen]).reshape(heads, dim)
            out[n, i], lse[n, :, i] = row.detach(), row_lse.detach()
            if dout is not None:
                do = dout[n, i].detach().cpu().double()
                total = total + (row * do).sum()
                with torch.no_grad():
                    dp = torch.einsum("hgd,jhd->hgj", do.view(-1, group, dim), v[n, :seen]).reshape(heads, seen)
                    ds = p * (dp.abs() + (do * row).sum(-1).abs()[:, None])
                    grouped = ds.view(-1, group, seen)
                    terms["dq"][n, i] = torch.einsum("hgj,jhd->hgd", grouped, k[n, :seen].abs()).reshape(heads, dim) * scale
                    terms["dk"][n, :seen] += torch.einsum("hgj,hgd->jhd", grouped, q[n, i].abs().view(-1, group, dim)) * scale
                    if bias is not None:
                        terms["dbias"].index_add_(0, m[(torch.arange(seen) - (first + i)).clamp(-reach, reach) + reach], ds.t().contiguous())
    if dout is None:
        return out, lse
    total.requires_grad_(True) if not total.requires_grad else None
    given = [t for t in leaves if t is not None]
    grads = torch.autograd.grad(total, given, allow_unused=True) if any(t.requires_grad for t in given) and total.grad_fn is not None else [None] * len(given)
    grads = [torch.zeros_like(t) if g is None else g for t, g in zip(given, grads)]
    return (out, lse, *grads, terms) if bias is not None else (out, lse, *grads, None, terms)


def rotate(x, gain, table, positions, eps=1e-6, interleaved=False):
    """x [rows, heads, dim], pairs as complex numbers."""
    x = x.double() if not x.requires_grad else x
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    if table is None:
        return x
    rot = 2 * table.shape[1]
    if x.shape[0] == 0:
        return x
    turn = torch.view_as_complex(table.double())[positions.long()][:, None]
    head, rest = x[..., :rot], x[..., rot:]
    pair = head.unflatten(-1, (rot // 2, 2)) if interleaved else head.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
    return torch.cat([(z if interleaved else z.transpose(-1, -2)).flatten(-2), rest], -1)


def keep_mask(rows, cols, p, seed, step, site, first_row=0):
    import numpy as np
    from oracle.philox import philox4x32
    calls = -(-cols // 4)
    q = (np.uint64(first_row) + np.arange(rows, dtype=np.uint64))[:, None] * np.uint64(calls) + np.arange(calls, dtype=np.uint64)[None]
    ctr = np.stack([q & np.uint64(0xFFFFFFFF), (q >> np.uint64(32)) | np.uint64(1 << 31), np.full_like(q, site), np.full_like(q, step)], -1)
    w = philox4x32(ctr, np.array([seed & 0xFFFFFFFF, seed >> 32], dtype=np.uint64)).reshape(rows, 4 * calls)[:, :cols]
    return torch.from_numpy(w.astype(np.float64) >= float(round(p * 2 ** 32)))
