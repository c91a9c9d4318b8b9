"""Plain 64-bit forms of the calls around the key / value cache, sequence by sequence, and the bounds of their rounding."""
import math

import torch


def attention(q, k, v, start, length, q_cu, groups=None, scale=None, skip=()):
    """(out, lse, weights added per cache row, sum p |v|, largest scale * sum |q k| of a row) in float64.  `groups`: list of
    (first sequence, last + 1, prefix start, prefix length).  Rows of the sequences in `skip` are NaN."""
    n_q, H, d = q.shape
    kv = k.shape[1]
    rep = H // kv
    scale = scale or 1.0 / math.sqrt(d)
    dev = q.device
    out = torch.full((n_q, H, d), float("nan"), dtype=torch.float64, device=dev)
    lse = torch.full((n_q, H), float("nan"), dtype=torch.float64, device=dev)
    pv = torch.zeros_like(out)
    size = torch.zeros_like(lse)
    weights = torch.zeros(k.shape[0], dtype=torch.float64, device=dev)
    for b in range(len(start)):
        r0, r1 = q_cu[b], q_cu[b + 1]
        if b in skip or r0 == r1:
            continue
        pre = torch.zeros(0, dtype=torch.long, device=dev)
        for b0, b1, ps, pl in groups or []:
            if b0 <= b < b1:
                pre = torch.arange(ps, ps + pl, device=dev)
        for t in range(r1 - r0):
            n_own = max(0, length[b] - (r1 - r0) + t + 1)
            idx = torch.cat([pre, torch.arange(start[b], start[b] + n_own, device=dev)])
            if idx.numel() == 0:
                out[r0 + t], lse[r0 + t] = 0.0, -math.inf
                continue
            qq = q[r0 + t].double().view(kv, rep, d)
            kk, vv = k[idx].double(), v[idx].double()
            x = torch.einsum("grd,jgd->grj", qq, kk) * scale
            size[r0 + t] = (torch.einsum("grd,jgd->grj", qq.abs(), kk.abs()) * abs(scale)).amax(-1).reshape(H)
            l = torch.logsumexp(x, -1)
            p = torch.exp(x - l[..., None])
            out[r0 + t] = torch.einsum("grj,jgd->grd", p, vv).reshape(H, d)
            pv[r0 + t] = torch.einsum("grj,jgd->grd", p, vv.abs()).reshape(H, d)
            lse[r0 + t] = l.reshape(H)
            weights[idx] += p.sum((0, 1)) / H
    return out, lse, weights, pv, size


def check_attention(got, lse, ref, dtype, n_keys):
    """Rounding of a correct result: every probability once to the element type (half a step, and half of its smallest subnormal
    relative to a largest probability of 1), the output once, and fp32 sums of up to a few thousand terms around that (2^-15)."""
    out, l, _, pv, size = ref
    half = torch.finfo(dtype).eps / 2
    sub = torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2
    tol = half * out.abs() + (half + 2.0 ** -15) * pv * (1 + 2.0 ** -7) + sub * (1 + 8.0 * n_keys)
    bad = ~((got.double() - out).abs() <= tol) & ~(torch.isnan(out) & torch.isnan(got))
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), ((got.double() - out).abs() / tol).nan_to_num(9e9).max().item())
    if lse is not None:
        # 128 products summed in fp32 (2^-24 * 128 of the sum of magnitudes), the sum of the probabilities, the logarithm
        tol = 2.0 ** -17 * size + 2.0 ** -18 * (1 + l.abs())
        fine = ((lse.double() - l).abs() <= tol) | ((l == -math.inf) & (lse == -math.inf)) | (torch.isnan(l) & torch.isnan(lse))
        assert fine.all(), (fine.logical_not().nonzero()[:4].tolist(), (lse.double() - l).abs().nan_to_num(0).max().item())


def check_weights(got, before, ref, n_rows):
    """p = exp(x - lse): twice the bound of a logit as a relative error; the sums and the last addition in fp32."""
    _, _, w, _, size = ref
    rel = 2.0 ** -15 * float(size.max()) + 2.0 ** -16
    want = before.double() + w
    tol = rel * w + 2.0 ** -23 * want.abs() + 2.0 ** -30 * n_rows
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), ((got.double() - want).abs() / tol).max().item())


def rank(weights, pos, n, sink, recent, newest):
    """Row numbers, best first (weights, pos: lists of one sequence)."""
    def key(i):
        if i < sink or pos[i] > newest - recent:
            return (0, 0.0, i)
        w = weights[i]
        return (2, 0.0, i) if w != w else (1, -(w + 0.0), i)
    return sorted(range(n), key=key)


def evict(weights, pos, keep, sink, recent):
    n = len(weights)
    if n <= keep:
        return list(range(n))
    return sorted(rank(weights, pos, n, sink, recent, max(pos))[:keep])


def rotate(x, pos, rot, layout, freq, magnitude=1.0, inverse=False):
    """x [rows, heads, d] rotated in float64; freq: radians per position of every pair (float64)."""
    n = rot // 2
    f = pos.double()[:, None, None] * freq.double()[None, None, :] * (-1.0 if inverse else 1.0)
    y = x.double().clone()
    a, b = (x[..., :n], x[..., n:rot]) if layout == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    a, b = a.double(), b.double()
    ra, rb = (a * f.cos() - b * f.sin()) * magnitude, (b * f.cos() + a * f.sin()) * magnitude
    if layout == "half":
        y[..., :n], y[..., n:rot] = ra, rb
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = ra, rb
    return y
