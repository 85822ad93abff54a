"""Token-mixer operators without a GPU: what the library and the binding refuse before anything is launched, and the oracle's
own definitions on small cases."""
import ctypes
import os
import re

import pytest

torch = pytest.importorskip("torch")
import paper_2512_18453_b200 as nv
from oracle import token_mixer as ref
from paper_2512_18453_b200 import token_mixer as tm

INVALID, UNSUPPORTED, CUDA = -1, -7, -8
P = 1 << 20                      # an address that nothing is launched with


def seqs(B=2, T=4, cu=0, slots=0, resume=0, n=2):
    return tm._Sequences(B, T, cu, slots, resume, n)


def conv(q=None, type=nv.token_mixer.F16, x=(P, 32, 128), w=P, b=0, D=32, W=4, state=P, y=(P + 4096, 32, 128), flags=0):
    q = seqs() if q is None else q
    x, y = tm._Rows(*x), tm._Rows(*y)
    return nv.lib().nova_causal_conv1d(ctypes.byref(q), type, ctypes.byref(x), w, b, D, W, state, ctypes.byref(y), flags, None)


def scan(q=None, type=nv.token_mixer.F16, **k):
    q = seqs() if q is None else q
    rows = {n: tm._Rows(P + 4096 * i, 32, 128) for i, n in enumerate(("u", "delta", "B", "C", "z", "y"))}
    a = dict(rows, B_group=0, C_group=0, A=P, D=P, delta_bias=P, state=P, channels=32, states=16, groups=1, flags=0)
    a.update(k)
    c = tm._Scan(*[a[f] for f, _ in tm._Scan._fields_])
    return nv.lib().nova_selective_scan(ctypes.byref(q), type, ctypes.byref(c), None)


def int4(type=nv.token_mixer.F16, x=P, x_row=64, M=2, K=64, codes=P, scales=P, zeros=0, group=32, b=0, N=8, y=P + 4096, y_row=8):
    return nv.lib().nova_linear_int4(type, x, x_row, M, K, codes, scales, zeros, group, b, N, y, y_row, None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="addresses that must not reach a kernel")
def test_good_arguments_get_as_far_as_the_missing_device():
    assert conv() == CUDA and scan() == CUDA and int4() == CUDA
    assert conv(seqs(T=1)) == CUDA and scan(seqs(T=1)) == CUDA
    assert conv(seqs(cu=P, slots=P, resume=P)) == CUDA and scan(seqs(cu=P, slots=P, resume=P)) == CUDA
    assert scan(D=0, delta_bias=0, state=0, z=tm._Rows(0, 0, 0)) == CUDA


@pytest.mark.parametrize("k", [
    dict(type=3), dict(type=-1), dict(D=0), dict(W=1), dict(W=5), dict(w=0), dict(w=P + 1), dict(b=P + 1), dict(state=P + 1), dict(flags=2),
    dict(x=(0, 32, 128)), dict(x=(P + 1, 32, 128)), dict(x=(P, -1, 128)), dict(x=(P, 32, -1)), dict(y=(P, 32, 128)), dict(y=(0, 0, 0)),
    dict(q=seqs(B=-1)), dict(q=seqs(T=-1)), dict(q=seqs(T=1 << 31)), dict(q=seqs(T=(1 << 31) - 8192)), dict(q=seqs(n=-1)), dict(q=seqs(cu=P + 2)), dict(q=seqs(slots=P + 2)),
    dict(state=0, q=seqs(slots=P)), dict(state=0, q=seqs(resume=P)), dict(q=seqs(B=(1 << 31) - 1), D=1 << 12),
])
def test_conv_refusals(k):
    assert conv(**k) == INVALID


@pytest.mark.parametrize("k", [
    dict(type=3), dict(channels=0), dict(states=0), dict(states=65), dict(groups=0), dict(groups=3), dict(A=0), dict(A=P + 2), dict(D=P + 2),
    dict(delta_bias=P + 1), dict(state=P + 2), dict(flags=1), dict(B_group=-1), dict(C_group=-1), dict(u=tm._Rows(0, 32, 128)), dict(z=tm._Rows(P + 1, 32, 128)),
    dict(B=tm._Rows(P, -2, 0)), dict(y=tm._Rows(P, 32, 128)), dict(y=tm._Rows(P + 4 * 4096, 32, 128)),
    dict(q=seqs(B=-1)), dict(q=seqs(T=-1)), dict(q=seqs(T=1 << 31)), dict(state=0, q=seqs(slots=P)), dict(q=seqs(B=(1 << 31) - 1), channels=1 << 12),
])
def test_scan_refusals(k):
    assert scan(**k) == INVALID


@pytest.mark.parametrize("k", [
    dict(type=3), dict(x=0), dict(x=P + 1), dict(codes=0), dict(codes=P + 8), dict(scales=0), dict(scales=P + 1), dict(b=P + 1), dict(y=0), dict(y=P), dict(M=0),
    dict(M=17), dict(N=0), dict(K=0), dict(K=48), dict(K=65), dict(group=16), dict(group=0), dict(group=256, K=256), dict(K=(1 << 17) + 32), dict(N=(1 << 26) + 1), dict(x_row=-1), dict(y_row=-1),
])
def test_int4_refusals(k):
    assert int4(**k) == INVALID


def test_int4_refuses_floats():
    assert int4(type=tm.F32) == UNSUPPORTED


def test_nothing_to_do_is_no_error():
    assert conv(seqs(B=0)) == 0 and conv(seqs(T=0)) == 0 and scan(seqs(B=0)) == 0 and scan(seqs(T=0)) == 0
    assert nv.lib().nova_causal_conv1d(None, 0, None, None, None, 1, 2, None, None, 0, None) == INVALID
    assert nv.lib().nova_selective_scan(None, 0, None, None) == INVALID


def test_binding_refuses_host_tensors_and_shapes():
    h = lambda *s: torch.zeros(*s, dtype=torch.float16)
    for call in (lambda: nv.causal_conv1d(h(1, 4, 8), h(8, 4)), lambda: nv.causal_conv1d_step(h(1, 8), h(1, 3, 8), h(8, 4)),
                 lambda: nv.causal_conv1d(torch.zeros(1, 4, 8, dtype=torch.int32), h(8, 4)), lambda: nv.causal_conv1d_step(h(1, 8), None, h(8, 4)),
                 lambda: nv.selective_scan(h(1, 4, 8), h(1, 4, 8), torch.zeros(8, 4), h(1, 4, 4), h(1, 4, 4)),
                 lambda: nv.selective_scan_step(h(1, 8), None, h(1, 8), torch.zeros(8, 4), h(1, 4), h(1, 4)),
                 lambda: nv.linear_int4(h(1, 32), torch.zeros(8, 16, dtype=torch.uint8), h(8, 1)),
                 lambda: nv.causal_conv1d(h(4, 8), h(8, 4)), lambda: nv.causal_conv1d(h(1, 4, 8), h(8, 4), cu_seqlens=torch.zeros(2, dtype=torch.int32)),
                 lambda: nv.causal_conv1d(h(4, 8), h(8, 4), cu_seqlens=torch.zeros(0, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()


def test_constants_and_structures_agree_with_the_header():
    text = open(os.path.join(os.path.dirname(__file__), "..", "include", "nova.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for name, value in (("NOVA_F32", tm.F32), ("NOVA_F16", tm.F16), ("NOVA_BF16", tm.BF16), ("NOVA_SILU", tm.SILU), ("NOVA_SOFTPLUS", tm.SOFTPLUS)):
        assert int(re.search(r"\b%s\s*=\s*(\d+)" % name, text).group(1)) == value
    assert int(re.search(r"NOVA_INT4_MAX_ROWS\s+(\d+)", text).group(1)) == nv.INT4_MAX_ROWS
    # natural alignment on both sides
    assert ctypes.sizeof(tm._Rows) == 24 and ctypes.sizeof(tm._Sequences) == 48
    assert ctypes.sizeof(tm._Scan) == 6 * 24 + 2 * 8 + 4 * 8 + 4 * 4


# ---------------------------------------------------------------- the oracle against independent forms
def test_oracle_convolution_is_the_library_convolution_in_64_bits():
    g = torch.Generator().manual_seed(1)
    x, w, b = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((9, 5), (5, 3), (5,)))
    ref.HALF_STEP[torch.float64] = ref.SUBNORMAL[torch.float64] = 0.0
    y, _, state = ref.causal_conv1d(x, w, b, ref.sequences(1, 9, nslots=1), torch.zeros(1, 2, 5, dtype=torch.float64))
    want = torch.nn.functional.conv1d(x.t()[None], w[:, None], b, padding=2, groups=5)[0, :, :9].t()
    assert torch.allclose(y, want, rtol=0, atol=1e-13) and torch.equal(state[0], x[-2:])


def test_oracle_scan_is_the_sum_over_all_pairs_of_tokens():
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    ref.HALF_STEP[torch.float64] = ref.SUBNORMAL[torch.float64] = 0.0
    T, D, N = 7, 3, 4
    u, delta, B, C, z, h0 = r(T, D), r(T, D).abs(), r(T, 1, N), r(T, 1, N), r(T, D), r(1, D, N)
    A, skip = -r(D, N).abs(), r(D)
    y, _, state, _ = ref.selective_scan(u, delta, A, B, C, ref.sequences(1, T, nslots=1), skip, z, None, False, h0)
    S = torch.cumsum(delta, 0)
    for t in range(T):
        h = torch.exp(S[t][:, None] * A) * h0[0]
        for s in range(t + 1):
            h = h + torch.exp((S[t] - S[s])[:, None] * A) * (delta[s] * u[s])[:, None] * B[s, 0]
        want = ((h * C[t, 0]).sum(1) + skip * u[t]) * torch.nn.functional.silu(z[t])
        assert torch.allclose(y[t], want, rtol=1e-12, atol=1e-12)
    assert torch.allclose(state[0], h, rtol=1e-12, atol=1e-12)


def test_oracle_int4_unpacks_low_bits_first():
    codes = torch.tensor([[0x21, 0xF8] + [0x88] * 14], dtype=torch.uint8)
    w = ref.int4_matrix(codes, torch.ones(1, 1), None)
    assert w[0, :4].tolist() == [-7.0, -6.0, 0.0, 7.0] and (w[0, 4:] == 0).all()


def test_oracle_sequences_follow_the_header():
    assert ref.sequences(3, 10, [-4, 3, 3, 20], [2, 0, 9], [True, False, True], 4) == [(0, 0, 3, 2, True)]
    assert ref.sequences(2, 5) == [(0, 0, 5, None, False), (1, 5, 10, None, False)]


def test_conv_refuses_more_channels_than_the_header_allows():
    most = 65535 * 256
    text = open(os.path.join(os.path.dirname(__file__), "..", "include", "nova.h")).read()
    assert re.search(r"NOVA_CONV1D_MAX_CHANNELS \((.*)\)", text).group(1) == "65535 * 256"
    wide = dict(x=(P, most + 1, 4 * most), y=(P + 4096, most + 1, 4 * most))
    assert conv(D=most + 1, **wide) == INVALID and conv(seqs(B=0), D=most, **wide) == 0
    if not torch.cuda.is_available():
        assert conv(D=most, **wide) == CUDA


def test_binding_tells_outputs_whose_rows_overlap():
    x, buf = torch.zeros(2, 5, 32, dtype=torch.float16), torch.zeros(4096, dtype=torch.float16)
    out = lambda strides, lead=(2, 5): tm._output(buf.as_strided((*lead, 32), (*strides, 1)), x, lead, 32)
    for strides in ((32, 32), (0, 32), (32, 0), (31, 500), (500, 31), (64, 32), (159, 32), (33, 64), (40, 71), (128, 32)):
        with pytest.raises(ValueError):
            out(strides)
    for strides in ((160, 32), (32, 64), (500, 40), (40, 72), (192, 40)):
        assert out(strides).stride()[:2] == strides
    assert out((0, 32), (1, 5)).shape == (1, 5, 32) and out((32, 0), (2, 1)).shape == (2, 1, 32) and out((32,), (5,)).shape == (5, 32)
    with pytest.raises(ValueError):
        out((31,), (5,))
