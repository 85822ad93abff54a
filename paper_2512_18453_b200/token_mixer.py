"""Operators of token mixers on torch tensors: causal_conv1d, selective_scan, linear_int4 and the single-token forms.

Argument marshalling only, like the rest of the binding; include/nova.h defines what each computes.  Tensors are on the
current device, calls go to its current stream.  Token tensors are [B, L, columns], or packed [rows, columns] with
`cu_seqlens` [B + 1] (int32, on the device); their columns are contiguous, the other strides are free, so that slices of
a projection's output are taken as they are.  ValueError for arguments of another kind, NovaError for what the library refuses.
"""
import ctypes

from .binding import NovaError, _check, _fast, _stream, lib

F32, F16, BF16 = 0, 1, 2
SILU, SOFTPLUS = 1, 2
INT4_MAX_ROWS = 16


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row", ctypes.c_int64), ("seq", ctypes.c_int64)]


class _Sequences(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int32), ("tokens", ctypes.c_int64), ("cu_seqlens", ctypes.c_void_p),
                ("slots", ctypes.c_void_p), ("resume", ctypes.c_void_p), ("state_slots", ctypes.c_int64)]


class _Scan(ctypes.Structure):
    _fields_ = [(k, _Rows) for k in ("u", "delta", "B", "C", "z", "y")] + [
        ("B_group", ctypes.c_int64), ("C_group", ctypes.c_int64), ("A", ctypes.c_void_p), ("D", ctypes.c_void_p),
        ("delta_bias", ctypes.c_void_p), ("state", ctypes.c_void_p), ("channels", ctypes.c_int32),
        ("states", ctypes.c_int32), ("groups", ctypes.c_int32), ("flags", ctypes.c_int32)]


_torch = None
_types = {}
_ext = None


def _fast_calls():
    """The C extension's functions (csrc/fastcall.c), or False without it.  They take well-formed arguments and return None
    for others, which the functions here then look at one by one."""
    global _ext
    if _ext is None:
        _init()
        _ext = _fast()
        if _ext:
            addr = lambda f: ctypes.cast(f, ctypes.c_void_p).value
            L = lib()
            _ext.bind_mixer(addr(L.nova_causal_conv1d), addr(L.nova_selective_scan), addr(L.nova_linear_int4), _torch.float32,
                            _torch.float16, _torch.bfloat16, _torch.int32, _torch.uint8, _torch.bool,
                            getattr(getattr(getattr(_torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None))
    return _ext


def _done(r, where):
    if type(r) is int:
        raise NovaError(r, where)
    return r


def _init():
    global _torch
    import torch
    _torch = torch
    _types.update({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})


def _type(x, name, allowed=(F32, F16, BF16)):
    if _torch is None:
        _init()
    t = _types.get(getattr(x, "dtype", None))
    if t not in allowed:
        raise ValueError("%s: a tensor of %s is needed" % (name, ", ".join(("float32", "float16", "bfloat16")[a] for a in allowed)))
    return t


def _here(t, name, dtype, shape=None):
    """Address of a tensor of `dtype` on the current device with contiguous columns, `shape` (None entries: any size)."""
    if not t.is_cuda or t.get_device() != _torch.cuda.current_device():
        raise ValueError("%s: not on the current CUDA device" % name)
    if t.dtype != dtype:
        raise ValueError("%s: %s is needed, not %s" % (name, dtype, t.dtype))
    if shape is not None and (t.dim() != len(shape) or any(b is not None and a != b for a, b in zip(t.shape, shape))):
        raise ValueError("%s: shape %s where %s is needed" % (name, tuple(t.shape), tuple("any" if b is None else b for b in shape)))
    return t.data_ptr()


def _whole(t, name, dtype, shape):
    p = _here(t, name, dtype, shape)
    if not t.is_contiguous():
        raise ValueError("%s: not contiguous" % name)
    return p


def _token_rows(t, name, dtype, lead, inner):
    """nova_rows of a token tensor [*lead, *inner]; lead is (rows,) or (sequences, tokens)."""
    p = _here(t, name, dtype, (*lead, *inner))
    st = t.stride()
    if t.shape[-1] > 1 and st[-1] != 1:
        raise ValueError("%s: the columns are not contiguous" % name)
    return _Rows(p, st[len(lead) - 1], st[0] if len(lead) == 2 else 0)


def _output(out, x, lead, D):
    if out is None:
        return _torch.empty((*lead, D), dtype=x.dtype, device=x.device)
    if out.dim() == len(lead) + 1:                     # rows that lie over each other would be written twice
        wide = D                                       # of what is repeated with the next larger stride
        for stride, n in sorted((out.stride(k), out.shape[k]) for k in range(len(lead)) if out.shape[k] > 1):
            if stride < wide:
                raise ValueError("out: its rows overlap")
            wide += (n - 1) * stride
    return out


def _sequences(x, step, cu_seqlens, slots, resume, state, name):
    """(nova_sequences, leading sizes of the token tensors)"""
    if step:
        if x.dim() != 2:
            raise ValueError("%s: [sequences, channels] is needed" % name)
        lead, B, L = (x.shape[0],), x.shape[0], 1
    elif cu_seqlens is None:
        if x.dim() != 3:
            raise ValueError("%s: [sequences, tokens, channels] is needed without cu_seqlens" % name)
        lead, B, L = (x.shape[0], x.shape[1]), x.shape[0], x.shape[1]
    else:
        if x.dim() != 2:
            raise ValueError("%s: [rows, channels] is needed with cu_seqlens" % name)
        lead, B, L = (x.shape[0],), cu_seqlens.numel() - 1, x.shape[0]
        if B < 0:
            raise ValueError("cu_seqlens: one value more than there are sequences is needed")
    if state is None and (slots is not None or resume is not None):
        raise ValueError("slots and resume belong to a state")
    q = _Sequences(B, L, 0, 0, 0, 0)
    if cu_seqlens is not None:
        q.cu_seqlens = _whole(cu_seqlens, "cu_seqlens", _torch.int32, (B + 1,))
    if state is not None:
        q.state_slots = state.shape[0]
        if slots is not None:
            q.slots = _whole(slots, "slots", _torch.int32, (B,))
        elif state.shape[0] < B:
            raise ValueError("state: fewer slots than sequences")
    if resume is not None:
        q.resume = _whole(resume, "resume", _torch.uint8 if resume.dtype == _torch.uint8 else _torch.bool, (B,))
    return q, lead


def _step_rows(r):
    """The row stride of a [sequences, columns] tensor is that of its sequences."""
    r.seq, r.row = r.row, 0
    return r


def _conv(x, state, weight, bias, cu_seqlens, slots, resume, silu, out, step):
    ext = _ext or _fast_calls()
    if ext:
        r = ext.causal_conv1d(x, state, weight, bias, cu_seqlens, slots, resume, SILU if silu else 0, out, step)
        if r is not None:
            return _done(r, "nova_causal_conv1d")
    type = _type(x, "x")
    q, lead = _sequences(x, step, cu_seqlens, slots, resume, state, "x")
    D, dtype = x.shape[-1], x.dtype
    w = _whole(weight, "weight", dtype, (D, None))
    W = weight.shape[1]
    b = None if bias is None else _whole(bias, "bias", dtype, (D,))
    s = None if state is None else _whole(state, "state", dtype, (None, W - 1, D))
    y = _output(out, x, lead, D)
    xr, yr = _token_rows(x, "x", dtype, lead, (D,)), _token_rows(y, "out", dtype, lead, (D,))
    if step:
        xr, yr = _step_rows(xr), _step_rows(yr)
    _check(lib().nova_causal_conv1d(ctypes.byref(q), type, ctypes.byref(xr), w, b, D, W, s, ctypes.byref(yr), SILU if silu else 0,
                                    _stream()), "nova_causal_conv1d")
    return y


def causal_conv1d(x, weight, bias=None, *, silu=False, state=None, cu_seqlens=None, slots=None, resume=None, out=None):
    """Causal convolution per channel of whole sequences.

    x [B, L, D] or packed [rows, D]; weight [D, W], W from 2 to 4; bias [D]; state [slots, W - 1, D] holds each sequence's
    last inputs, oldest first, and is updated in place; slots [B] (int32) names each sequence's slot (default: its number),
    one outside the state marks padding; resume [B] (bool) says which sequences start from their slot (default: all)."""
    return _conv(x, state, weight, bias, cu_seqlens, slots, resume, silu, out, False)


def causal_conv1d_step(x, state, weight, bias=None, *, silu=False, slots=None, out=None):
    """causal_conv1d of one token for each sequence: x [B, D] -> [B, D]; state is updated in place."""
    if state is None:
        raise ValueError("state: needed for a single token")
    return _conv(x, state, weight, bias, None, slots, None, silu, out, True)


def _scan(u, state, delta, A, B, C, D, z, delta_bias, softplus, cu_seqlens, slots, resume, out, step):
    ext = _ext or _fast_calls()
    if ext:
        r = ext.selective_scan(u, state, delta, A, B, C, D, z, delta_bias, cu_seqlens, slots, resume, SOFTPLUS if softplus else 0, out, step)
        if r is not None:
            return _done(r, "nova_selective_scan")
    type = _type(u, "u")
    q, lead = _sequences(u, step, cu_seqlens, slots, resume, state, "u")
    dtype, f32 = u.dtype, _torch.float32
    c = _Scan()
    c.channels = u.shape[-1]
    c.A = _whole(A, "A", f32, (c.channels, None))
    c.states = A.shape[1]
    c.D = None if D is None else _whole(D, "D", f32, (c.channels,))
    c.delta_bias = None if delta_bias is None else _whole(delta_bias, "delta_bias", f32, (c.channels,))
    c.state = None if state is None else _whole(state, "state", f32, (None, c.channels, c.states))
    c.flags = SOFTPLUS if softplus else 0
    grouped = B.dim() == len(lead) + 2
    c.groups = B.shape[-2] if grouped else 1
    inner = (c.groups, c.states) if grouped else (c.states,)
    y = _output(out, u, lead, c.channels)
    for k, t in (("u", u), ("delta", delta), ("z", z), ("y", y)):
        if t is not None:
            setattr(c, k, _token_rows(t, "out" if k == "y" else k, dtype, lead, (c.channels,)))
    for k, t in (("B", B), ("C", C)):
        setattr(c, k, _token_rows(t, k, dtype, lead, inner))
    if grouped:
        c.B_group, c.C_group = B.stride(-2), C.stride(-2)
    if step:
        for k in ("u", "delta", "z", "y", "B", "C"):
            _step_rows(getattr(c, k))
    _check(lib().nova_selective_scan(ctypes.byref(q), type, ctypes.byref(c), _stream()), "nova_selective_scan")
    return y


def selective_scan(u, delta, A, B, C, *, D=None, z=None, delta_bias=None, softplus=False, state=None, cu_seqlens=None,
                   slots=None, resume=None, out=None):
    """Selective scan of whole sequences.

    u, delta, z [B, L, D] or packed [rows, D]; A [D, N] float32; B, C [.., N], or [.., G, N] with G groups of channels;
    D, delta_bias [D] float32; state [slots, D, N] float32, updated in place; slots and resume as for causal_conv1d."""
    return _scan(u, state, delta, A, B, C, D, z, delta_bias, softplus, cu_seqlens, slots, resume, out, False)


def selective_scan_step(u, state, delta, A, B, C, *, D=None, z=None, delta_bias=None, softplus=False, slots=None, out=None):
    """selective_scan of one token for each sequence: token tensors are [B, columns]; state is updated in place."""
    if state is None:
        raise ValueError("state: needed for a single token")
    return _scan(u, state, delta, A, B, C, D, z, delta_bias, softplus, None, slots, None, out, True)


def linear_int4(x, codes, scales, zeros=None, bias=None, *, out=None):
    """x [M, K] (half or bfloat16, M up to INT4_MAX_ROWS) times 4-bit weights -> [M, N].

    codes [N, K / 2] uint8, even k in the low four bits; scales [N, K / group] of x's type, group 32, 64 or 128;
    zeros [N, K / group] uint8 (default 8 everywhere); bias [N] of x's type."""
    ext = _ext or _fast_calls()
    if ext:
        r = ext.linear_int4(x, codes, scales, zeros, bias, out)
        if r is not None:
            return _done(r, "nova_linear_int4")
    type = _type(x, "x", (F16, BF16))
    if x.dim() != 2 or codes.dim() != 2 or scales.dim() != 2:
        raise ValueError("x, codes and scales have two dimensions")
    M, K = x.shape
    N, groups = scales.shape
    group = K // groups if groups and K % groups == 0 else 0
    xr = _token_rows(x, "x", x.dtype, (M,), (K,))
    c = _whole(codes, "codes", _torch.uint8, (N, K // 2))
    s = _whole(scales, "scales", x.dtype, (N, groups))
    z = None if zeros is None else _whole(zeros, "zeros", _torch.uint8, (N, groups))
    b = None if bias is None else _whole(bias, "bias", x.dtype, (N,))
    y = _output(out, x, (M,), N)
    yr = _token_rows(y, "out", x.dtype, (M,), (N,))
    _check(lib().nova_linear_int4(type, xr.data, xr.row, M, K, c, s, z, group, b, N, yr.data, yr.row, _stream()), "nova_linear_int4")
    return y
