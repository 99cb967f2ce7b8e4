"""The token layers' C ABI on the host: what descriptors and arguments are
refused, and the sizes that the queries report.  No GPU: every call here ends
before it would enqueue anything."""
import ctypes

import pytest

from paper_2204_03418_amd import coinf as C

P = 0x1000  # a pointer that is never followed


def conv(**more):
    d = dict(batch=2, channels=8, kernel=4, has_bias=1, act=C.CO_ACT_SILU, dtype=C.CO_F32)
    d.update(more)
    return C.ShortConvDesc(*(d[k] for k, _ in C.ShortConvDesc._fields_))


def scan(**more):
    d = dict(batch=2, heads=4, head_dim=16, state_size=32, groups=2, dt_softplus=1,
             dtype=C.CO_BF16, dt_dtype=C.CO_BF16)
    d.update(more)
    return C.ScanDesc(*(d[k] for k, _ in C.ScanDesc._fields_))


def norm(**more):
    d = dict(batch=2, tokens=3, dim=16, groups=2, gate=0, residual=0, dtype=C.CO_F32,
             residual_dtype=C.CO_F32, eps=1e-5)
    d.update(more)
    return C.NormDesc(*(d[k] for k, _ in C.NormDesc._fields_))


def ref(v):
    return ctypes.byref(v)


def test_queries():
    n = C.i64()
    assert C.co_shortconv_query(ref(conv()), ref(n)) == C.CO_OK and n.value == 2 * 3 * 8 * 4
    assert C.co_shortconv_query(ref(conv(kernel=1, dtype=C.CO_BF16)), ref(n)) == C.CO_OK
    assert n.value == 0
    assert C.co_scan_query(ref(scan()), ref(n)) == C.CO_OK and n.value == 2 * 4 * 16 * 32 * 4
    assert C.co_scan_query(ref(scan()), None) == C.CO_EINVAL
    assert C.co_shortconv_query(None, ref(n)) == C.CO_EINVAL


@pytest.mark.parametrize("bad", [
    dict(batch=0), dict(channels=0), dict(kernel=0), dict(kernel=9), dict(act=3), dict(act=-1),
    dict(dtype=2), dict(batch=1 << 30, channels=1 << 30)], ids=str)
def test_shortconv_descriptors_refused(bad):
    n = C.i64()
    assert C.co_shortconv_query(ref(conv(**bad)), ref(n)) == C.CO_EINVAL


@pytest.mark.parametrize("bad", [
    dict(batch=0), dict(heads=0), dict(head_dim=0), dict(state_size=0), dict(state_size=257),
    dict(groups=0), dict(groups=3), dict(dtype=5), dict(dt_dtype=-1),
    dict(heads=1 << 16, head_dim=1 << 16, groups=1),
    dict(batch=1 << 20, heads=1 << 10, head_dim=1 << 10)], ids=str)
def test_scan_descriptors_refused(bad):
    n = C.i64()
    assert C.co_scan_query(ref(scan(**bad)), ref(n)) == C.CO_EINVAL
    assert C.co_scan_workspace_bytes(ref(scan(**bad)), 100, ref(n)) == C.CO_EINVAL


def call_conv(d, x=(P, 80, 8), y=(2 * P, 80, 8), T=10, weight=P, bias=P, lengths=None, state=P):
    c = C.ShortConvCall(weight, bias, C.Tokens(*x), C.Tokens(*y), lengths, state, T, 1)
    return C.co_shortconv_forward_steps(ref(d), ref(c), None)


def test_shortconv_arguments():
    assert call_conv(conv(), T=0) == C.CO_OK                      # nothing to do
    assert call_conv(conv(), T=-1) == C.CO_EINVAL
    assert call_conv(conv(), weight=None) == C.CO_EINVAL
    assert call_conv(conv(), bias=None) == C.CO_EINVAL
    assert call_conv(conv(), x=(None, 80, 8)) == C.CO_EINVAL
    assert call_conv(conv(), x=(P + 2, 80, 8)) == C.CO_EINVAL     # not a float's address
    assert call_conv(conv(), x=(P, -80, 8)) == C.CO_EINVAL
    assert call_conv(conv(), x=(P, 80, 1 << 60)) == C.CO_EINVAL
    assert call_conv(conv(), y=(P, 80, 8)) == C.CO_EINVAL         # in place
    assert call_conv(conv(), y=(2 * P, 80, 7)) == C.CO_EINVAL     # tokens overlap
    assert call_conv(conv(), y=(2 * P, 79, 8)) == C.CO_EINVAL     # streams overlap
    assert call_conv(conv(), y=(2 * P, 8, 15)) == C.CO_EINVAL     # token-major, overlapping
    assert call_conv(conv(), lengths=P + 1) == C.CO_EINVAL
    assert call_conv(conv(batch=1 << 16, channels=1 << 12), x=(P, 0, 0), y=(2 * P, 1 << 42, 1 << 12),
                     T=1 << 30) == C.CO_EINVAL                    # too many values


def call_scan(d, T=10, A=P, ws=None, nws=0, state=P, **io):
    t = dict(x=(P, 640, 64), dt=(P, 40, 4), b=(P, 640, 64), c=(P, 640, 64), y=(2 * P, 640, 64))
    t.update(io)
    c = C.ScanCall(A, None, None, *(C.Tokens(*t[k]) for k in ("x", "dt", "b", "c", "y")), None,
                   state, ws, nws, T, 1)
    return C.co_scan_forward_steps(ref(d), ref(c), None)


def test_scan_arguments():
    assert call_scan(scan(), T=0) == C.CO_OK
    for bad in (dict(T=-1), dict(A=None), dict(nws=-1), dict(x=(None, 640, 64)),
                dict(dt=(P + 1, 40, 4)), dict(b=(P, 640, -1)), dict(y=(P, 640, 64)),
                dict(y=(2 * P, 640, 63)), dict(y=(2 * P, 639, 64)), dict(state=P + 2),
                dict(ws=P + 4, nws=1 << 20)):
        assert call_scan(scan(), **bad) == C.CO_EINVAL, bad
    assert C.co_scan_forward_steps(ref(scan()), None, None) == C.CO_EINVAL
    assert C.co_scan_forward_steps(None, ref(C.ScanCall()), None) == C.CO_EINVAL


def test_scan_workspace():
    """None for a few tokens; for long calls what the segments and chunks need,
    growing no faster than the tokens."""
    n = C.i64()
    d = scan(batch=1, heads=64, head_dim=64, state_size=128, groups=1)
    sizes = []
    for T in (0, 1, 4, 64, 1000, 16384, 1 << 20):
        assert C.co_scan_workspace_bytes(ref(d), T, ref(n)) == C.CO_OK
        sizes.append(n.value)
    assert sizes[:3] == [0, 0, 0] and 0 < sizes[3] < sizes[4] < sizes[5] < sizes[6]
    # decays of a chunk of 32 tokens and a head: 656 bytes; B . C: 3 tiles of 64 lanes; states of
    # at most 64 parts
    chunks = 1 << 15
    most = chunks * (64 * 656 + 3 * 64 * 16) + 64 * 64 * (64 * 128 + 1) * 4
    assert sizes[6] <= most
    assert C.co_scan_workspace_bytes(ref(d), -1, ref(n)) == C.CO_EINVAL
    assert C.co_scan_workspace_bytes(ref(d), 5, None) == C.CO_EINVAL


def call_norm(d, x=(P, 48, 16), gate=None, residual=None, y=(P, 48, 16), out=None, weight=P,
              scale=None):
    t = [C.Tokens(*v) if v else C.Tokens() for v in (x, gate, residual, y, out)]
    return C.co_norm_forward(ref(d), ref(C.NormCall(*t, weight, scale)), None)


def test_norm_arguments():
    assert call_norm(norm(batch=0)) == C.CO_OK and call_norm(norm(tokens=0), x=None) == C.CO_OK
    for bad in (dict(dim=0), dict(groups=3), dict(groups=0), dict(gate=3), dict(residual=-1),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(dtype=7),
                dict(residual_dtype=7), dict(batch=-1), dict(tokens=-1)):
        assert call_norm(norm(**bad)) == C.CO_EINVAL, bad
    assert call_norm(norm(dim=2 * 32769)) == C.CO_ENOTSUP
    assert call_norm(norm(batch=1 << 20, tokens=1 << 10)) == C.CO_ENOTSUP
    assert call_norm(norm(gate=1)) == C.CO_EINVAL                 # no gate given
    assert call_norm(norm(residual=1), residual=(P, 48, 16)) == C.CO_EINVAL  # no place for the sum
    assert call_norm(norm(), y=None) == C.CO_EINVAL
    assert call_norm(norm(), y=(P, 48, 15)) == C.CO_EINVAL
    assert call_norm(norm(), x=(P + 1, 48, 16)) == C.CO_EINVAL
    assert call_norm(norm(), weight=P + 1) == C.CO_EINVAL


def test_host_only_layers_refuse_host_tensors():
    import torch

    with pytest.raises(ValueError):
        C.CoShortConv(torch.ones(8, 4), batch=1)
    with pytest.raises(ValueError):
        C.CoScan(torch.ones(4), batch=1, head_dim=8, state_size=8)
    with pytest.raises(ValueError):
        C.CoNorm(torch.ones(8))
    with pytest.raises(ValueError):
        C.CoNorm()
