"""The operators on rows of channels in 64 bits, sequence by sequence, each with a bound on what fp32 arithmetic may be off.

A function returns pairs (value, bound).  u = 2^-24 is the relative error of one fp32 rounding; the bounds carry
the magnitudes that enter every sum, so that cancellation is allowed for where it happens and nowhere else.
"""
import math

import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def lengths_of(cu):
    return [b - a for a, b in zip(cu[:-1], cu[1:])]


def check(got, want, what, rows=None):
    """|got - value| <= bound + half a step of the stored type, element by element."""
    value, bound = want
    g = got.detach().double().cpu().reshape(value.shape)
    if rows is not None:
        g, value, bound = g[:rows], value[:rows], bound[:rows]
    # two bounds meet: the value before rounding is off by `bound`, and rounding it is relative to that value
    room = bound + HALF_STEP[got.dtype] * (value.abs() + bound) + 1e-37
    off = (g - value).abs()
    bad = ~(off <= room)
    assert not bad.any(), (what, int(bad.sum()), "of", bad.numel(), "worst", float((off / room).nan_to_num(float("inf")).max()),
                           "first at", bad.nonzero()[0].tolist())


def scan(x, g, lens, init, complement, dout=None, dfin=None):
    """x, g [N, C]; init, dfin [S, C] or None.  Returns out, final (and dx, dgate, dinit)."""
    x, g = x.double().cpu(), g.double().cpu()
    N, C = x.shape
    S = len(lens)
    init = torch.zeros(S, C, dtype=torch.float64) if init is None else init.double().cpu()
    a, keep = g.exp(), -torch.expm1(g)
    b = x * keep if complement else x
    # one step: the factor (6 u of a: series, scaling, its form), the product and the sum, and what a blocked order
    # adds by forming a h once more from the sum of the gates (|sum| u <= 40 u where the factor is not negligible)
    K = 64 * U
    out, before, e_out, e_before = (torch.zeros(N, C, dtype=torch.float64) for _ in range(4))
    final, e_final = init.clone(), torch.zeros_like(init)
    at = 0
    for s, n in enumerate(lens):
        h, e, m = init[s].clone(), torch.zeros(C, dtype=torch.float64), init[s].abs()
        for t in range(at, at + n):
            before[t], e_before[t] = h, e
            h = a[t] * h + b[t]
            m = a[t] * m + b[t].abs()
            e = a[t] * e + K * m
            out[t], e_out[t] = h, e
        final[s], e_final[s] = h, e
        at += n
    got = [(out, e_out), (final, e_final)]
    if dout is None:
        return got
    dout = dout.double().cpu()
    dfin = torch.zeros(S, C, dtype=torch.float64) if dfin is None else dfin.double().cpu()
    dx, dg, e_dx, e_dg = (torch.zeros(N, C, dtype=torch.float64) for _ in range(4))
    dinit, e_dinit = dfin.clone(), torch.zeros_like(dfin)
    at = 0
    for s, n in enumerate(lens):
        c, e, m = dfin[s].clone(), torch.zeros(C, dtype=torch.float64), dfin[s].abs()   # a_{t+1} dh_{t+1}
        for t in range(at + n - 1, at - 1, -1):
            dh, mh, eh = dout[t] + c, dout[t].abs() + m, e + U * (dout[t].abs() + m)
            dx[t] = dh * keep[t] if complement else dh
            e_dx[t] = (eh + K * mh) * (keep[t] if complement else 1.0)
            c, m = a[t] * dh, a[t] * mh
            e = a[t] * eh + K * m
            u = before[t] - x[t] if complement else before[t]
            mu = before[t].abs() + (x[t].abs() if complement else 0.0)
            dg[t] = u * c
            e_dg[t] = e_before[t] * c.abs() + u.abs() * e + e_before[t] * e + 4 * U * mu * c.abs()
        dinit[s], e_dinit[s] = c, e
        at += n
    return got + [(dx, e_dx), (dg, e_dg), (dinit, e_dinit)]


def conv(x, w, bias, lens, init, silu, quick, dout=None, dfin=None, chain=None):
    """x [N, C], w [C, W]; init, dfin [S, W-1, C] or None.  `quick`: the fast exponential and division (bf16).  `chain`: additions
    that a term of the weights' sums goes through at most (without it: any order of the N terms)."""
    x, w = x.double().cpu(), w.double().cpu()
    N, C = x.shape
    W, S = w.shape[1], len(lens)
    b = torch.zeros(C, dtype=torch.float64) if bias is None else bias.double().cpu()
    init = torch.zeros(S, W - 1, C, dtype=torch.float64) if init is None else init.double().cpu()
    out, e_out = torch.zeros(N, C, dtype=torch.float64), torch.zeros(N, C, dtype=torch.float64)
    final = torch.zeros(S, W - 1, C, dtype=torch.float64)
    grads = dout is not None
    dfin = torch.zeros(S, W - 1, C, dtype=torch.float64) if dfin is None else dfin.double().cpu()
    dx, e_dx = torch.zeros(N, C, dtype=torch.float64), torch.zeros(N, C, dtype=torch.float64)
    dinit, e_dinit = torch.zeros_like(final), torch.zeros_like(final)
    dw, m_dw, e_dw = (torch.zeros(C, W, dtype=torch.float64) for _ in range(3))
    db, m_db, e_db = (torch.zeros(C, dtype=torch.float64) for _ in range(3))
    S_ERR = 2.0 ** -19 if quick else 8 * U      # sigmoid, relative (the argument's rounding: |z| u, z below 88)
    at = 0
    for s, n in enumerate(lens):
        ext = torch.cat([init[s], x[at:at + n]])
        final[s] = ext[n:]
        win = ext.unfold(0, W, 1)[:n] if n else ext.new_zeros(0, C, W)      # [n, C, W]
        z = (win * w).sum(-1) + b
        ez = (W + 1) * U * ((win * w).abs().sum(-1) + b.abs())
        sig = torch.sigmoid(z)
        e_sig = (S_ERR + z.abs() * U) * sig + 0.25 * ez
        if silu:
            out[at:at + n], e_out[at:at + n] = z * sig, 1.1 * ez + z.abs() * (S_ERR + z.abs() * U) * sig + 2 * U * (z * sig).abs()
        else:
            out[at:at + n], e_out[at:at + n] = z, ez
        if grads:
            d = dout[at:at + n].double().cpu()
            if silu:
                slope = sig * (1 + z * (1 - sig))
                # |slope'| <= 1/2; the fast sigmoid's error enters with 1 + |z|
                e_slope = 0.5 * ez + (1 + z.abs()) * 2 * e_sig + 4 * U * sig * (1 + z.abs())
            else:
                slope, e_slope = torch.ones_like(z), torch.zeros_like(z)
            dz, e_dz = d * slope, d.abs() * e_slope + U * (d * slope).abs()
            de, m_de, e_de = (torch.zeros(n + W - 1, C, dtype=torch.float64) for _ in range(3))
            for i in range(W):
                de[i:i + n] += w[:, i] * dz
                m_de[i:i + n] += (w[:, i] * dz).abs()
                e_de[i:i + n] += w[:, i].abs() * e_dz
                dw[:, i] += (dz * win[..., i]).sum(0)
                m_dw[:, i] += (dz * win[..., i]).abs().sum(0)
                e_dw[:, i] += (e_dz * win[..., i].abs()).sum(0)
            de[n:] += dfin[s]
            m_de[n:] += dfin[s].abs()
            e_de += (W + 2) * U * m_de
            dinit[s], e_dinit[s] = de[:W - 1], e_de[:W - 1]
            dx[at:at + n], e_dx[at:at + n] = de[W - 1:], e_de[W - 1:]
            db += dz.sum(0)
            m_db += dz.abs().sum(0)
            e_db += e_dz.sum(0)
        at += n
    got = [(out, e_out), (final, torch.zeros_like(final))]
    if not grads:
        return got
    terms = (N + 64 if chain is None else chain) * U
    return got + [(dx, e_dx), (dw, e_dw + terms * m_dw), (db, e_db + terms * m_db), (dinit, e_dinit)]


def norm(x, w, kind, eps, angle, layout, dy=None, chain=None):
    """x [N, H, D]; w [D] or None; angle [N, R/2] in fp64 or None.  Returns y (and dx, dw).  `chain`: as of conv, of the N H terms."""
    x = x.double().cpu()
    N, H, D = x.shape
    wt = torch.ones(D, dtype=torch.float64) if w is None else w.double().cpu()
    share = 1.0 / D if kind == "rms" else 1.0
    r = (x.square().sum(-1, keepdim=True) * share + eps) ** -0.5
    u = x * r
    E = 24 * U                                  # of r: eight and five sums, the fma, two steps of rsqrtf, products
    A = 2.0 ** -20                              # of a sine or cosine: the angle's fp32 remainder (pi 2^-24) and two steps

    def turned(v, e, sign):
        if angle is None:
            return v, e
        m = angle.shape[1]
        c, s = torch.cos(angle)[:, None].cpu(), sign * torch.sin(angle)[:, None].cpu()
        first = slice(0, m) if layout == "half" else slice(0, 2 * m, 2)
        second = slice(m, 2 * m) if layout == "half" else slice(1, 2 * m, 2)
        p, q, ep, eq = v[..., first], v[..., second], e[..., first], e[..., second]
        y, ey = v.clone(), e.clone()
        y[..., first], y[..., second] = p * c - q * s, p * s + q * c
        room = (A + 2 * U) * (p.abs() + q.abs())
        ey[..., first], ey[..., second] = ep * c.abs() + eq * s.abs() + room, ep * s.abs() + eq * c.abs() + room
        return y, ey

    y, ey = turned(u * wt, E * (u * wt).abs(), 1.0)
    if dy is None:
        return [(y, ey)]
    dv, e_dv = turned(dy.double().cpu(), torch.zeros(N, H, D, dtype=torch.float64), -1.0)
    du, e_du = dv * wt, e_dv * wt.abs() + U * (dv * wt).abs()
    dot = (du * u).sum(-1, keepdim=True) * share
    m_dot = (du * u).abs().sum(-1, keepdim=True) * share
    e_dot = (e_du * u.abs()).sum(-1, keepdim=True) * share + (E + 16 * U) * m_dot
    dx = r * (du - u * dot)
    e_dx = r * (e_du + u.abs() * e_dot + (E + 8 * U) * (du.abs() + u.abs() * m_dot))
    dw = (dv * u).sum((0, 1))
    e_dw = (e_dv * u.abs()).sum((0, 1)) + (E + (N * H + 64 if chain is None else chain) * U) * (dv * u).abs().sum((0, 1))
    return [(y, ey), (dx, e_dx), (dw, e_dw)]


def angles(positions, inv_freq):
    """In 64 bits; reduced by whole turns with the product's own rounding (2^-53 of it) as the only loss."""
    return torch.remainder(positions.double().cpu()[:, None] * inv_freq.double().cpu(), 2 * math.pi)
