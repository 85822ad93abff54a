"""Token-mixer operators in 64 bits, token by token, with bounds on what a float evaluation may be off.

Tensors are torch tensors on any device.  Each function returns the value and, per element, the largest error of an
evaluation that carries its sums in float (unit u = 2^-24) and rounds the output once to the storage type.
"""
import torch

U = 2.0 ** -24
# half a step of a type relative to the value, and half a step of its subnormals
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# A float below 2^-126 has fewer bits, or none where an instruction flushes it: what it stands for is off by up to 2^-126,
# whatever its relative rounding.  That holds for each of dt, dt u, dt u B, a term of the state and a term of y.
TINY = 2.0 ** -126
SUBNORMAL = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def rounded(value, error, dtype):
    """Bound after the one rounding of a value known to within `error`."""
    return error + HALF_STEP[dtype] * (value.abs() + error) + SUBNORMAL[dtype]


def sequences(count, tokens, cu=None, slots=None, resume=None, nslots=None):
    """[(sequence, first row, row behind the last, slot or None, resumes)], what the header says of bounds and padding applied."""
    out = []
    for i in range(count):
        lo, hi = (i * tokens, (i + 1) * tokens)
        if cu is not None:
            lo = min(max(int(cu[i]), 0), tokens)
            hi = min(max(int(cu[i + 1]), lo), tokens)
        slot = None
        if nslots is not None:
            slot = i if slots is None else int(slots[i])
            if not 0 <= slot < nslots:
                continue
        if hi > lo:
            out.append((i, lo, hi, slot, slot is not None and (resume is None or bool(resume[i]))))
    return out


def silu(v, e):
    """v sigmoid(v) and its bound: the slope is below 1.1; exponential, sum, quotient and the product 8 (1 + |v|) u relative."""
    y = v * torch.sigmoid(v)
    return y, 1.1 * e + 8 * (1 + v.abs()) * U * y.abs()


def causal_conv1d(x, weight, bias, seqs, state=None, act=False):
    """x [rows, D], weight [D, W] -> (y, bound, state): y of the rows of `seqs`, NaN elsewhere; state as it is left."""
    dtype, f = x.dtype, lambda a: a.double()
    D, W = weight.shape
    y = torch.full(x.shape, float("nan"), dtype=torch.float64, device=x.device)
    bound = torch.zeros_like(y)
    state = None if state is None else state.clone()
    for _, lo, hi, slot, resume in seqs:
        old = state[slot] if resume else x.new_zeros(W - 1, D)
        row = torch.cat([old, x[lo:hi]])
        v = torch.zeros(hi - lo, D, dtype=torch.float64, device=x.device)
        size = torch.zeros_like(v)
        if bias is not None:
            v, size = v + f(bias), size + f(bias).abs()
        for k in range(W):
            p = f(row[k:k + hi - lo]) * f(weight)[:, k]
            v, size = v + p, size + p.abs()
        e = (W + 1) * U * size
        if act:
            v, e = silu(v, e)
        y[lo:hi], bound[lo:hi] = v, rounded(v, e, dtype)
        if slot is not None:
            state[slot] = row[hi - lo:]
    return y, bound, state


def selective_scan(u, delta, A, B, C, seqs, D=None, z=None, delta_bias=None, softplus=False, state=None):
    """u, delta, z [rows, channels], B, C [rows, groups, states] -> (y, its bound, state, its bound).

    The error of a state follows the state's own recurrence: a step multiplies it by the decay and adds what the step's own
    roundings leave.  Relative to their factors: dt 4u (softplus: exponential, logarithm, sum), dt A another 2u, so that the
    decay is off by (6 |dt A| + 4) u, a product and a sum 2u more; the input dt u B by 7u.  The bound takes 8 for each."""
    dtype, f = u.dtype, lambda a: a.double()
    ch = u.shape[1]
    A = A.clamp(-torch.finfo(torch.float32).max, torch.finfo(torch.float32).max)         # as the header says of infinities
    at = torch.arange(ch, device=u.device) // (ch // B.shape[1])
    y = torch.full(u.shape, float("nan"), dtype=torch.float64, device=u.device)
    bound = torch.zeros_like(y)
    state = None if state is None else f(state).clone()
    sbound = None if state is None else torch.zeros_like(state)
    dt_all = f(delta) if delta_bias is None else f(delta) + f(delta_bias)
    # of the bias and the softplus' argument: a rounding that is absolute, not relative, in dt
    dt_abs = U * (dt_all.abs() + f(delta).abs()) if delta_bias is not None else torch.zeros_like(dt_all)
    if softplus:
        slope = torch.sigmoid(dt_all)
        dt_all, dt_abs = torch.logaddexp(dt_all, torch.zeros_like(dt_all)), dt_abs * slope + TINY
    for _, lo, hi, slot, resume in seqs:
        h = state[slot] if resume else torch.zeros(ch, A.shape[1], dtype=torch.float64, device=u.device)
        e, size = torch.zeros_like(h), h.abs()
        for t in range(lo, hi):
            dt, da = dt_all[t][:, None], dt_abs[t][:, None]
            ut, Bt, Ct = f(u[t])[:, None], f(B[t])[at], f(C[t])[at]
            arg = dt * f(A)
            a, b = torch.exp(arg), dt * ut * Bt
            e = a * e + (8 * U * (1 + arg.abs()) + da * f(A).abs()) * a * size + 8 * U * b.abs() + da * (ut * Bt).abs() + TINY * (2 + Bt.abs())
            h, size = a * h + b, a * size + b.abs()
            v, ve = (h * Ct).sum(1), (Ct.abs() * (e + (A.shape[1] + 4) * U * size) + TINY).sum(1)
            if D is not None:
                v, ve = v + f(D) * ut[:, 0], ve + 2 * U * ((f(D) * ut[:, 0]).abs() + (h * Ct).abs().sum(1))
            if z is not None:
                gate, ge = silu(f(z[t]), 0.0)
                v, ve = v * gate, ve * gate.abs() + (v.abs() + ve) * (ge + U * gate.abs())
            y[t], bound[t] = v, rounded(v, ve, dtype)
        if slot is not None:
            state[slot], sbound[slot] = h, e + U * size + TINY
    return y, bound, state, sbound


def int4_matrix(codes, scales, zeros, dtype=torch.float64):
    """The weights that codes, scales and zeros stand for."""
    N, half = codes.shape
    group = 2 * half // scales.shape[1]
    q = torch.stack([codes & 15, codes >> 4], -1).reshape(N, 2 * half).to(dtype)
    per = lambda a: a.to(dtype).repeat_interleave(group, 1)
    return (q - (8.0 if zeros is None else per(zeros & 15))) * per(scales)


def linear_int4(x, codes, scales, zeros=None, bias=None):
    """(y, bound).  Codes less zeros and their products with x are exact; the sums run over `group` products and over the groups,
    in any order, each partial sum off by 2 u of the sum of magnitudes."""
    w = int4_matrix(codes, scales, zeros)
    y, size = x.double() @ w.t(), x.double().abs() @ w.abs().t()
    terms = x.shape[1] / 16 + 32
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return y, rounded(y, 2 * U * terms * size, x.dtype)
