"""The operators on sequences and the 8-bit matrix form from their definitions, in 64 bits on the CPU, each with a bound on
what float arithmetic may be off by.

U is half a step of float (2^-24).  A bound counts the roundings of the definition's own operations in any order; the
hardware's exponential, logarithm and reciprocal are within one unit in the last place, 2 U each.
"""
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def spans(count, tokens, start=None, length=None):
    """First row and number of rows of every sequence."""
    out = []
    for i in range(count):
        b, e = (start[i], start[i + 1]) if start is not None else (i * (tokens // count), (i + 1) * (tokens // count))
        n = e - b
        if length is not None:
            n = max(0, min(n, length[i]))
        out.append((b, n))
    return out


def silu(v, err):
    """v * sigmoid(v) and its bound: the slope is at most 1.1; exponent's argument |v| * 2 U, exp, add, reciprocal, product."""
    y = v * torch.sigmoid(v)
    return y, 1.1 * err + (8 + 2 * v.abs()) * U * y.abs()


def causal_conv(x, filt, bias, state, rows, source, target, act, out, dtype):
    """(output, its bound, state): `out` and `state` are what the call found there, in 64 bits."""
    x, filt = x.double(), filt.double()
    W = filt.shape[1]
    out, state, old = out.double().clone(), state.double().clone(), state.double().clone()
    bound = torch.zeros_like(out)
    for i, (b, n) in enumerate(rows):
        if n == 0:
            continue
        before = old[source[i]] if 0 <= source[i] < len(old) else torch.zeros_like(old[0])
        full = torch.cat([before, x[b:b + n]])
        y = torch.zeros(n, x.shape[1], dtype=torch.float64) + (0 if bias is None else bias.double())
        size = y.abs()
        for k in range(W):
            y = y + full[k:k + n] * filt[:, k]
            size = size + (full[k:k + n] * filt[:, k]).abs()
        err = (W + 1) * U * size
        if act:
            y, err = silu(y, err)
        out[b:b + n], bound[b:b + n] = y, err + half_step(dtype) * (y.abs() + err)
        if 0 <= target[i] < len(state):
            state[target[i]] = full[n:]
    return out, bound, state


def selective_scan(x, dt, A, B, C, D, z, dt_bias, state, rows, source, target, groups, softplus, out, dtype, piece=0):
    """(output, bound, state, bound).  `piece`: rows over which a decay may be taken from a sum of steps, whose roundings
    grow with it."""
    d = lambda t: None if t is None else t.double()  # noqa: E731
    x, dt, A, B, C, D, z, dt_bias = map(d, (x, dt, A, B, C, D, z, dt_bias))
    N, per = A.shape[1], A.shape[0] // groups
    out, state, old = d(out).clone(), d(state).clone(), d(state).clone()
    bound, sbound = torch.zeros_like(out), torch.zeros_like(state)
    v = dt + (0 if dt_bias is None else dt_bias)
    dv = U * v.abs()                                        # the sum with the bias
    if softplus:
        delta = torch.nn.functional.softplus(v, threshold=1e9)
        ddelta = dv * torch.sigmoid(v) + (10 + 2 * v.abs()) * U * delta
    else:
        delta, ddelta = v, dv
    for i, (b, n) in enumerate(rows):
        if n == 0:
            continue
        h = old[source[i]].clone() if 0 <= source[i] < len(old) else torch.zeros_like(old[0])
        E = torch.zeros_like(h)
        for t in range(b, b + n):
            Bt, Ct = (m[t].view(groups, 1, N).expand(-1, per, -1).reshape(groups * per, N) for m in (B, C))
            step = delta[t][:, None] * A
            a = torch.exp(step)
            # the decay's relative error: the exponential and its product, and its argument's roundings
            da = 4 * U + (4 + piece) * U * step.abs() + ddelta[t][:, None] * A.abs()
            add = (delta[t] * x[t])[:, None] * Bt
            dadd = 4 * U * add.abs() + (ddelta[t] * x[t].abs())[:, None] * Bt.abs()
            E = a * E + (a * h).abs() * da + dadd
            h = a * h + add
            E = E + U * h.abs()
            y = (Ct * h).sum(1)
            err = (Ct.abs() * E).sum(1) + (N + 4) * U * (Ct * h).abs().sum(1)
            if D is not None:
                y = y + D * x[t]
                err = err + 2 * U * (D * x[t]).abs() + U * y.abs()
            if z is not None:
                g, dg = silu(z[t], torch.zeros_like(z[t]))
                err = err * g.abs() + y.abs() * dg + U * (y * g).abs()
                y = y * g
            out[t], bound[t] = y, err + half_step(dtype) * (y.abs() + err)
        if 0 <= target[i] < len(state):
            state[target[i]], sbound[target[i]] = h, E
    return out, bound, state, sbound


def quantize(x, block_rows):
    """(codes [rows, 128 * blocks] of float8_e4m3fn, scales [blocks of columns, blocks of rows]): the definition's own single-precision
    steps, so that they have to be met exactly."""
    M, K = x.shape
    kb, mb = -(-K // 128), -(-M // block_rows)
    full = torch.zeros(mb * block_rows, kb * 128, dtype=torch.float32)
    full[:M, :K] = x.float()
    v = full.view(mb, block_rows, kb, 128)
    most = torch.where(v.isnan(), 0.0, v.abs()).amax((1, 3))
    scales = torch.where(most > 0, (most / 448.0).clamp(min=2.0 ** -126), torch.ones(()))
    q = (v / scales[:, None, :, None]).view(mb * block_rows, kb * 128)[:M].clamp(-448.0, 448.0)
    return q.to(torch.float8_e4m3fn), scales.t().contiguous()


def matmul(a, a_scales, b, b_scales, bias, dtype):
    """(output, bound).  Products of e4m3 values are exact in float (two 4-bit mantissas).  Float output: every one of a
    block's 128 additions may round (twice half a step: the matrix units need not round to nearest), the block's result
    is scaled and added once.  bfloat16 output: the e4m3 instruction cuts every product of 8 neighbours to 13 bits below the
    leading bit of the largest, which loses less than 2^-13 of that largest for each of the 7 others; the largest of 8 products is at most
    the product of the 8 largest factors."""
    A = a.double() * a_scales.double().t().repeat_interleave(128, 1)
    B = b.double() * b_scales.double().t().repeat_interleave(128, 1).repeat_interleave(128, 0)[:b.shape[0]]
    y, size = A @ B.t(), A.abs() @ B.abs().t()
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    err = (128 + 2 * a_scales.shape[0] + 4) * 2 * U * size
    if dtype == torch.bfloat16:
        eights = lambda m: m.abs().view(m.shape[0], -1, 8).amax(2)  # noqa: E731
        err = err + 7 * 2.0 ** -13 * (eights(A) @ eights(B).t())
    return y, err + half_step(dtype) * (y.abs() + err)


def check(name, got, want, bound):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, name
    off = (got - want).abs() - bound
    bad = ~(off <= 0)
    assert not bad.any(), (name, int(bad.sum()), bad.nonzero()[0].tolist(), got[bad][0].item(), want[bad][0].item(),
                           bound[bad][0].item())
