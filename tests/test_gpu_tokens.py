"""The token layers (short convolution, selective scan, norm) against plain
64-bit forms: sizes on and off the tiles, every dtype, strides and unaligned
slices, lengths with empty streams, NaN past them, states carried over pieces.

Bounds.  A float32 sum of n terms is off by at most about n 2^-24 of the sum of
their magnitudes (`size`), each elementary function here by a few units; an
output is then rounded once to its dtype (unit roundoff u).  The scan's chunked
form in bfloat16 also rounds the factors of its products over a chunk to
bfloat16 once, an error of at most u `size`.
"""
import numpy as np
import pytest
import torch

import token_ref as R
from paper_2204_03418_amd import coinf

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16
U = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def randn(g, *shape, scale=1.0, dtype=F32):
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def lengths_for(kind, g, B, T):
    if kind == "full":
        return None
    n = torch.randint(0, T + 1, (B,), generator=g)
    n[0] = 0
    if B > 1:
        n[1] = T
    if B > 2:
        n[2] = min(1, T)
    return n.to(torch.int32)


def put(t, pad=0, shift=0):
    """t (B, T, ...) on the device as a slice of a wider tensor: `pad` values
    more a token, from `shift` values on; NaN around it."""
    if pad == 0:
        return t.to(DEV)
    B, T = t.shape[:2]
    n = t[0, 0].numel() if B and T else int(np.prod(t.shape[2:]))
    wide = torch.full((B, T, n + pad), float("nan"), dtype=t.dtype, device=DEV)
    s = wide[:, :, shift:shift + n]
    s.copy_(t.reshape(B, T, n))
    return s.unflatten(-1, tuple(t.shape[2:])) if t.dim() > 3 else s


def poison(t, lengths):
    """NaN in the tokens past the lengths."""
    if lengths is not None:
        for i, n in enumerate(lengths.tolist()):
            t[i, n:] = float("nan")
    return t


# ------------------------------------------------------------ short convolution

CONV = [
    # B, T, C, K, dtype, act, lengths, pad, shift
    (1, 1, 8, 4, BF16, "silu", "full", 0, 0),
    (3, 1, 24, 3, F32, "silu", "ragged", 0, 0),
    (4, 1, 33, 2, BF16, "none", "ragged", 0, 0),
    (2, 5, 432, 4, BF16, "silu", "ragged", 0, 0),
    (2, 8, 40, 8, F32, "relu", "full", 16, 8),
    (3, 9, 264, 4, BF16, "silu", "ragged", 16, 8),
    (3, 65, 264, 4, BF16, "silu", "ragged", 3, 1),
    (2, 130, 100, 5, F32, "silu", "ragged", 0, 0),
    (4, 64, 256, 3, BF16, "none", "full", 0, 0),
    (2, 77, 7, 1, F32, "silu", "ragged", 0, 0),
    (2, 77, 16, 1, BF16, "relu", "full", 0, 0),
    (5, 3, 48, 6, F32, "silu", "ragged", 0, 0),
    (5, 2, 48, 7, BF16, "silu", "ragged", 0, 0),
    (1, 300, 1, 4, F32, "silu", "full", 0, 0),
]


@pytest.mark.parametrize("case", CONV, ids=str)
@pytest.mark.parametrize("bias", [True, False])
def test_shortconv(case, bias):
    B, T, C, K, dtype, act, kind, pad, shift = case
    g = gen(7)
    x, w = randn(g, B, T, C, dtype=dtype), randn(g, C, K, scale=K ** -0.5, dtype=dtype)
    bs = randn(g, C, dtype=dtype) if bias else None
    state = randn(g, B, K - 1, C, dtype=dtype)
    n = lengths_for(kind, g, B, T)
    xd = put(poison(x.clone(), n), pad, shift)
    nd = None if n is None else n.to(DEV)
    layer = coinf.CoShortConv(w.to(DEV), None if bs is None else bs.to(DEV), batch=B, act=act,
                              state=state.clone().to(DEV))
    got = layer.forward_steps(xd, nd, update_state=False)
    assert torch.equal(layer.state.cpu(), state)
    again = layer.forward_steps(xd, nd)
    assert torch.equal(got, again)
    y, size, new = R.shortconv(R.np64(x), R.np64(w), R.np64(bs), R.np64(state), n, act)
    # K + 1 terms; exp2, its argument, reciprocal and product: 8 units more
    R.within(got, y, U[dtype] * np.abs(y) + (K + 9) * R.U32 * size, f"conv {case}")
    assert np.array_equal(R.np64(layer.state), new)             # inputs, not computed
    clean = layer.forward(xd, nd)
    y, size, _ = R.shortconv(R.np64(x), R.np64(w), R.np64(bs), None, n, act)
    R.within(clean, y, U[dtype] * np.abs(y) + (K + 9) * R.U32 * size, f"conv clip {case}")


def test_shortconv_pieces_equal_clip():
    """Definition 1: a clip, pieces and single tokens have the same bits."""
    g = gen(8)
    for dtype in (F32, BF16):
        B, T, C, K = 2, 37, 72, 4
        x, w = randn(g, B, T, C, dtype=dtype).to(DEV), randn(g, C, K, dtype=dtype).to(DEV)
        layer = coinf.CoShortConv(w, batch=B)
        clip = layer.forward(x)
        out, t = [], 0
        for n in (1, 1, 2, 11, 1, 20, 1):
            out.append(layer.forward_steps(x[:, t:t + n]) if n > 1
                       else layer.forward_step(x[:, t])[:, None])
            t += n
        assert torch.equal(torch.cat(out, 1), clip)


# ------------------------------------------------------------ selective scan

SCAN = [
    # B, T, H, P, G, N, dtype, lengths, softplus, D, pad, shift
    (1, 1, 8, 64, 1, 16, F32, "full", True, True, 0, 0),
    (3, 1, 4, 64, 2, 128, BF16, "ragged", True, True, 8, 8),
    (2, 1, 3, 20, 1, 20, F32, "ragged", False, False, 0, 0),
    (2, 1, 2, 33, 2, 50, BF16, "full", True, True, 3, 1),
    (4, 1, 64, 64, 4, 128, BF16, "ragged", True, True, 0, 0),
    (2, 6, 8, 64, 8, 64, BF16, "ragged", True, True, 0, 0),
    (2, 5, 2, 128, 1, 256, F32, "full", True, True, 0, 0),
    (2, 16, 4, 64, 1, 128, BF16, "ragged", True, True, 0, 0),
    (2, 17, 4, 32, 2, 32, F32, "ragged", True, False, 0, 0),
    (1, 63, 2, 64, 1, 64, BF16, "full", True, True, 0, 0),
    (1, 64, 2, 64, 1, 64, F32, "full", True, True, 0, 0),
    (2, 65, 2, 48, 1, 128, BF16, "ragged", True, True, 16, 8),
    (3, 150, 6, 40, 3, 20, F32, "ragged", True, True, 0, 0),
    (3, 150, 5, 24, 5, 33, BF16, "ragged", True, True, 5, 3),
    (2, 200, 3, 64, 1, 256, BF16, "ragged", False, True, 0, 0),
    (2, 130, 2, 96, 2, 256, F32, "ragged", True, True, 0, 0),
    (1, 300, 4, 1, 1, 1, F32, "full", True, False, 0, 0),
    (2, 100, 12, 16, 2, 16, BF16, "ragged", True, True, 0, 0),
    (1, 900, 4, 64, 2, 128, BF16, "full", True, True, 0, 0),
    (2, 700, 3, 64, 1, 64, F32, "ragged", True, True, 0, 0),
    (1, 777, 1, 128, 1, 32, BF16, "full", True, True, 0, 0),
]


def scan_inputs(case, seed, dt_dtype=None):
    B, T, H, P, G, N, dtype = case[:7]
    g = gen(seed)
    silu = torch.nn.functional.silu
    step = torch.exp(torch.rand(H, generator=g) * 4.6 - 6.9)          # 0.001 .. 0.1
    v = dict(x=silu(randn(g, B, T, H, P)).to(dtype), b=silu(randn(g, B, T, G, N)).to(dtype),
             c=silu(randn(g, B, T, G, N)).to(dtype), A=-(torch.rand(H, generator=g) * 15 + 1),
             D=randn(g, H), state=randn(g, B, H, P, N, scale=0.3))
    if case[8]:
        v["dt"] = randn(g, B, T, H, scale=0.7).to(dt_dtype or dtype)
        v["dt_bias"] = torch.log(torch.expm1(step))
    else:
        v["dt"] = (torch.rand(B, T, H, generator=g) * 0.1).to(dt_dtype or dtype)
        v["dt_bias"] = None
    return v, lengths_for(case[7], g, B, T)


def scan_layer(case, v, state):
    B, T, H, P, G, N, dtype, _, softplus, skip = case[:10]
    return coinf.CoScan(v["A"].to(DEV), batch=B, head_dim=P, state_size=N, groups=G,
                        D=v["D"].to(DEV) if skip else None,
                        dt_bias=None if v["dt_bias"] is None else v["dt_bias"].to(DEV),
                        dt_softplus=softplus, dtype=dtype,
                        state=None if state is None else state.clone().to(DEV))


def scan_ref(case, v, state, n):
    return R.scan(R.np64(v["x"]), R.np64(v["dt"]), R.np64(v["b"]), R.np64(v["c"]), R.np64(v["A"]),
                  R.np64(v["D"]) if case[9] else None, R.np64(v["dt_bias"]), case[8],
                  R.np64(state), n)


def check_scan(case, got, state, ref, what):
    y, size, S, M = ref
    T, N, dtype = case[1], case[5], case[6]
    # a state is a sum over at most T tokens whose decays are products of as many factors of
    # a few units each, an output one over N values of it
    f32 = (4 * T + N + 64) * R.U32
    factors = U[dtype] if dtype is BF16 else 0.0
    R.within(got, y, U[dtype] * np.abs(y) + (factors + f32) * size, f"scan y {what}")
    R.within(state, S, f32 * M, f"scan state {what}")
    # roundings to nearest of random values: u / sqrt(3) at the most for the output, and as
    # much for the factors; float32 sums stay under 1e-5
    assert R.relative(got, y) <= (np.sqrt(2 / 3) * U[BF16] if dtype is BF16 else 1e-5)
    assert R.relative(state, S) <= 1e-5


@pytest.mark.parametrize("case", SCAN, ids=str)
def test_scan(case):
    B, T, H, P, G, N, dtype, kind, softplus, skip, pad, shift = case
    v, n = scan_inputs(case, 11)
    dev = {k: put(poison(v[k].clone(), n), pad, shift) for k in ("x", "b", "c", "dt")}
    nd = None if n is None else n.to(DEV)
    layer = scan_layer(case, v, v["state"])
    got = layer.forward_steps(dev["x"], dev["dt"], dev["b"], dev["c"], nd, update_state=False)
    assert torch.equal(layer.state.cpu(), v["state"])
    again = layer.forward_steps(dev["x"], dev["dt"], dev["b"], dev["c"], nd)
    assert torch.equal(got, again)
    check_scan(case, got, layer.state, scan_ref(case, v, v["state"], n), str(case))
    if n is not None:
        for i, k in enumerate(n.tolist()):
            assert not got[i, k:].any()
            if k == 0:
                assert torch.equal(layer.state[i].cpu(), v["state"][i])
    clean = layer.forward(dev["x"], dev["dt"], dev["b"], dev["c"], nd)
    y, size, _, _ = scan_ref(case, v, None, n)
    f32 = (4 * T + N + 64) * R.U32 + (U[dtype] if dtype is BF16 else 0.0)
    R.within(clean, y, U[dtype] * np.abs(y) + f32 * size, f"scan clip {case}")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_pieces_equal_clip(dtype):
    """Pieces of any length and single tokens reach the clip's outputs and state."""
    case = (2, 333, 4, 64, 2, 64, dtype, "full", True, True)
    v, _ = scan_inputs(case, 12)
    d = {k: v[k].to(DEV) for k in ("x", "dt", "b", "c")}
    layer = scan_layer(case, v, None)
    out, t = [], 0
    for n in (1, 1, 7, 64, 1, 130, 100, 29):
        p = {k: a[:, t:t + n] for k, a in d.items()}
        out.append(layer.forward_steps(p["x"], p["dt"], p["b"], p["c"]) if n > 1 else
                   layer.forward_step(*(p[k][:, 0] for k in ("x", "dt", "b", "c")))[:, None])
        t += n
    assert t == 333
    check_scan(case, torch.cat(out, 1), layer.state, scan_ref(case, v, None, None), "pieces")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [1, 5, 200])
def test_scan_float32_steps_beside_any_dtype(dtype, T):
    case = (2, T, 4, 32, 1, 48, dtype, "full", True, True)
    v, _ = scan_inputs(case, 13, dt_dtype=F32)
    layer = scan_layer(case, v, v["state"])
    got = layer.forward_steps(*(v[k].to(DEV) for k in ("x", "dt", "b", "c")))
    check_scan(case, got, layer.state, scan_ref(case, v, v["state"], None), "float32 dt")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [4, 200])
def test_scan_resets_and_standstill(dtype, T):
    """Decays to nothing (dt A far below any float32's logarithm, as a reset
    writes it) and none at all (dt = 0: a token that changes nothing): what
    follows a reset depends on it and its successors alone."""
    case = (2, T, 4, 32, 2, 32, dtype, "full", False, True)
    v, _ = scan_inputs(case, 14)
    v["dt"][:, 2::7] = 0.0
    v["dt"][:, T // 2] = 1e4
    v["x"][:, T // 2] *= 1e-4
    v["A"][1] = 0.0                                             # a head that never forgets
    v["dt"][:, T // 2, 1] = 0.01
    layer = scan_layer(case, v, v["state"])
    got = layer.forward_steps(*(v[k].to(DEV) for k in ("x", "dt", "b", "c")))
    check_scan(case, got, layer.state, scan_ref(case, v, v["state"], None), "resets")


def test_scan_token_major_and_broadcast_inputs():
    """(T, B, ...) tensors seen as (B, T, ...), and B and C that all streams share."""
    case = (3, 90, 4, 32, 1, 32, BF16, "full", True, True)
    v, _ = scan_inputs(case, 15)
    v["b"], v["c"] = v["b"][:1].expand(3, -1, -1, -1), v["c"][:1].expand(3, -1, -1, -1)
    layer = scan_layer(case, v, v["state"])
    turn = {k: v[k].to(DEV).transpose(0, 1).contiguous().transpose(0, 1) for k in ("x", "dt")}
    b, c = (v[k][:1].to(DEV).expand(3, -1, -1, -1) for k in ("b", "c"))
    out = torch.empty(90, 3, 4, 32, dtype=BF16, device=DEV).transpose(0, 1)
    got = layer.forward_steps(turn["x"], turn["dt"], b, c, out=out)
    assert got is out
    check_scan(case, got, layer.state, scan_ref(case, v, v["state"], None), "orders")


# ------------------------------------------------------------ norm

NORM = [
    # rows, dim, groups, x dtype, residual dtype, pad
    (1, 8, 1, BF16, BF16, 0),
    (5, 7, 1, F32, F32, 0),
    (64, 2048, 1, BF16, F32, 0),
    (33, 432, 3, F32, F32, 0),
    (10, 432, 2, BF16, BF16, 40),
    (9, 520, 1, BF16, F32, 3),
    (4, 4096, 1, BF16, BF16, 8),
    (3, 4100, 4, F32, BF16, 0),
    (3, 8192, 1, F32, F32, 0),
    (3, 8190, 1, BF16, F32, 0),
    (2, 16384, 1, BF16, BF16, 0),
    (2, 9001, 1, F32, F32, 0),
]


@pytest.mark.parametrize("case", NORM, ids=str)
@pytest.mark.parametrize("gate", [None, "before", "after"])
@pytest.mark.parametrize("residual", [None, "before", "after"])
def test_norm(case, gate, residual):
    rows, dim, groups, dtype, rdtype, pad = case
    g = gen(21)
    x, z = randn(g, rows, dim, dtype=dtype), randn(g, rows, dim, dtype=dtype)
    r = randn(g, rows, dim, scale=3.0, dtype=rdtype)
    w, s = randn(g, dim), randn(g, dim)
    w = w if dim % 3 else None
    wide = lambda t: put(t[None], pad, pad // 2)[0]  # noqa: E731
    layer = coinf.CoNorm(None if w is None else w.to(DEV), dim=dim, eps=1e-5, groups=groups,
                         gate=gate, residual=residual, scale=s.to(DEV) if residual else None)
    got = layer.forward(wide(x), gate=wide(z) if gate else None,
                        residual=wide(r) if residual else None)
    y, new = R.norm(R.np64(x), R.np64(z) if gate else None, R.np64(r) if residual else None,
                    R.np64(w), R.np64(s) if residual else None, groups, 1e-5, gate, residual)
    # a mean of squares over `width` values of one sign: its relative error is at most
    # width / 32 + 16 units (sums of up to 32 values in a lane, then in a tree), halved by the
    # root; the pre-norm's sum may cancel, by at most its own magnitude
    units = (32 + 24) * R.U32
    if residual == "after":
        size = np.abs(R.np64(r)) + np.abs(new - R.np64(r))
        R.within(got, new, U[rdtype] * np.abs(new) + units * size, f"norm {case} {gate}")
        return
    got_y, got_r = got if residual else (got, None)
    size = np.abs(y)
    if residual:
        a = R.np64(x) * (R.np64(z) * R.sigmoid(R.np64(z)) if gate == "before" else 1.0)
        mag = np.abs(R.np64(r)) + np.abs(R.np64(s) * a)
        R.within(got_r, new, U[rdtype] * np.abs(new) + 12 * R.U32 * mag, f"sum {case} {gate}")
        rms = np.sqrt((new.reshape(rows, groups, -1) ** 2).mean(-1) + 1e-5)
        after = np.abs(R.np64(z) * R.sigmoid(R.np64(z))) if gate == "after" else 1.0
        size = size + (mag / np.repeat(rms, dim // groups, 1)
                       * (1.0 if w is None else np.abs(R.np64(w))) * after)
    R.within(got_y, y, U[dtype] * np.abs(y) + units * size, f"norm {case} {gate} {residual}")


def test_norm_in_place_and_zero_rows():
    g = gen(22)
    x, z = randn(g, 2, 3, 96, dtype=BF16).to(DEV), randn(g, 2, 3, 96, dtype=BF16).to(DEV)
    r = randn(g, 2, 3, 96).to(DEV)
    x[0, 1] = 0.0
    layer = coinf.CoNorm(torch.ones(96, device=DEV), gate="before")
    want = layer.forward(x, gate=z)
    assert torch.equal(layer.forward(x.clone(), gate=z), want) and not want[0, 1].any()
    y = x.clone()
    assert torch.equal(layer.forward(y, gate=z, out=y), want)
    pre = coinf.CoNorm(dim=96, residual="before")
    y, new = pre.forward(x, residual=r)
    keep = r.clone()
    y2, same = pre.forward(x, residual=keep, residual_out=keep)
    assert same is keep and torch.equal(keep, new) and torch.equal(y2, y)
    none = pre.forward(x[:0], residual=r[:0])
    assert none[0].shape == (0, 3, 96)
    none = pre.forward(x[0, :0], residual=r[0, :0])
    assert none[1].shape == (0, 96)


def test_norm_axes():
    """Any number of leading axes, pieces of longer tensors, tokens before streams."""
    g = gen(23)
    x, z = randn(g, 3, 8, 64, dtype=BF16).to(DEV), randn(g, 3, 8, 100, dtype=BF16).to(DEV)
    layer = coinf.CoNorm(torch.ones(64, device=DEV), gate="after")
    want = layer.forward(x, gate=z[..., :64].contiguous())
    assert torch.equal(layer.forward(x, gate=z[..., :64]), want)
    assert torch.equal(layer.forward(x[:, 2:5], gate=z[:, 2:5, :64]), want[:, 2:5])
    assert torch.equal(layer.forward(x[1, 4], gate=z[1, 4, :64]), want[1, 4])
    assert torch.equal(layer.forward(x.view(3, 2, 4, 64), gate=z[..., :64].unflatten(1, (2, 4))),
                       want.view(3, 2, 4, 64))
    turn = x.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty_like(turn)
    assert torch.equal(layer.forward(turn, gate=z[..., :64], out=out), want)
    with pytest.raises(ValueError):
        layer.forward(x.transpose(0, 1).unflatten(0, (2, 4)),
                      gate=z[..., :64].transpose(0, 1).unflatten(0, (2, 4)).transpose(0, 2))


# ------------------------------------------------------------ refusals, streams, graphs


def test_refusals():
    w = torch.ones(8, 4, device=DEV)
    conv = coinf.CoShortConv(w, batch=2)
    x = torch.zeros(2, 5, 8, device=DEV)
    for bad in (x.cpu(), x.bfloat16(), x[:, :, :7], x[:1], x.transpose(1, 2), x[0]):
        with pytest.raises(ValueError):
            conv.forward_steps(bad)
    for n in (torch.ones(2), torch.ones(2, dtype=torch.int32), torch.ones(3, dtype=torch.int32)):
        with pytest.raises(ValueError):
            conv.forward_steps(x, n if n.numel() == 2 else n.to(DEV))
    with pytest.raises(coinf.CoinfError):
        conv.forward_steps(x, out=x)                            # not in place
    with pytest.raises(coinf.CoinfError):
        conv.forward_steps(x, out=torch.zeros(1, 5, 8, device=DEV).expand(2, -1, -1))
    with pytest.raises(coinf.CoinfError):
        coinf.CoShortConv(torch.ones(8, 9, device=DEV), batch=1)
    with pytest.raises(ValueError):
        coinf.CoShortConv(w, batch=2, state=torch.zeros(2, 4, 8, device=DEV))
    A = -torch.ones(4, device=DEV)
    scan = coinf.CoScan(A, batch=2, head_dim=8, state_size=8, groups=2, dtype=F32)
    v = dict(x=torch.zeros(2, 5, 4, 8, device=DEV), dt=torch.zeros(2, 5, 4, device=DEV),
             b=torch.zeros(2, 5, 2, 8, device=DEV), c=torch.zeros(2, 5, 2, 8, device=DEV))
    scan.forward_steps(**v)
    for k, bad in (("x", v["x"].bfloat16()), ("x", v["x"][:, :4]), ("dt", v["dt"].double()),
                   ("b", v["b"][:, :, :1]), ("c", v["c"].transpose(2, 3)), ("x", v["x"].cpu())):
        with pytest.raises(ValueError):
            scan.forward_steps(**{**v, k: bad})
    with pytest.raises(coinf.CoinfError):
        scan.forward_steps(**v, out=v["x"])
    for more in (dict(groups=3), dict(state_size=257), dict(head_dim=0)):
        with pytest.raises(coinf.CoinfError):
            coinf.CoScan(A, **{**dict(batch=2, head_dim=8, state_size=8, dtype=F32), **more})
    with pytest.raises(ValueError):
        coinf.CoScan(A, batch=2, head_dim=8, state_size=8, D=torch.ones(3, device=DEV))
    r = torch.zeros(3, 16, device=DEV)
    norm = coinf.CoNorm(torch.ones(16, device=DEV), gate="before")
    for args in (dict(x=r), dict(x=r, gate=r[:2]), dict(x=r, gate=r.bfloat16()),
                 dict(x=r[:, :8], gate=r[:, :8]), dict(x=r, gate=r, residual=r)):
        with pytest.raises(ValueError):
            norm.forward(**args)
    with pytest.raises(ValueError):
        coinf.CoNorm(torch.ones(16, device=DEV), groups=3)
    with pytest.raises(coinf.CoinfError):
        coinf.CoNorm(dim=32769).forward(torch.zeros(1, 32769, device=DEV))


def test_nothing_to_do():
    """No tokens: no outputs, the state as it was."""
    conv = coinf.CoShortConv(torch.ones(8, 4, device=DEV), batch=2)
    conv.state.fill_(3.0)
    assert conv.forward_steps(torch.zeros(2, 0, 8, device=DEV)).shape == (2, 0, 8)
    scan = coinf.CoScan(-torch.ones(4, device=DEV), batch=2, head_dim=8, state_size=8, dtype=F32)
    scan.state.fill_(3.0)
    e = [torch.zeros(2, 0, *s, device=DEV) for s in ((4, 8), (4,), (1, 8), (1, 8))]
    assert scan.forward_steps(*e).shape == (2, 0, 4, 8)
    assert (conv.state == 3).all() and (scan.state == 3).all()


@pytest.mark.parametrize("T", [1, 300])
def test_graph_replays_advance_the_states(T):
    """A captured call has no host counter: each replay takes the next tokens."""
    case = (2, T, 4, 64, 2, 64, BF16, "full", True, True)
    v, _ = scan_inputs(case, 31)
    x = v["x"].flatten(2).to(DEV)
    conv = coinf.CoShortConv(torch.full((256, 4), 0.25, dtype=BF16, device=DEV), batch=2)
    scan = scan_layer(case, v, v["state"])
    norm = coinf.CoNorm(torch.ones(256, device=DEV), gate="before")
    dt, b, c = (v[k].to(DEV) for k in ("dt", "b", "c"))

    def step():
        u = conv.forward_steps(x)
        y = scan.forward_steps(u.unflatten(-1, (4, 64)), dt, b, c)
        return norm.forward(y.flatten(2), gate=x)

    side = torch.cuda.Stream()
    start = conv.state.clone(), scan.state.clone()
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step()
    torch.cuda.synchronize()
    conv.state.copy_(start[0]), scan.state.copy_(start[1])
    got = []
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        got.append((out.clone(), scan.state.clone(), conv.state.clone()))
        x.mul_(-1.0)                                            # other tokens the next time
    x.copy_(v["x"].flatten(2))
    conv.state.copy_(start[0]), scan.state.copy_(start[1])
    for y, s, k in got:
        assert torch.equal(step(), y) and torch.equal(scan.state, s) and torch.equal(conv.state, k)
        x.mul_(-1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_scan_nonfinite_tokens_stay_behind(dtype, bad):
    """What is not finite at a token reaches no output before it, no other
    stream and no other row of its head."""
    case = (2, 150, 2, 32, 1, 32, dtype, "full", True, True)
    v, _ = scan_inputs(case, 41)
    y, size, S, M = scan_ref(case, v, v["state"], None)
    v["x"][0, 83, 1, 5] = bad
    layer = scan_layer(case, v, v["state"])
    got = layer.forward_steps(*(v[k].to(DEV) for k in ("x", "dt", "b", "c")))
    mark = torch.zeros(got.shape, dtype=torch.bool, device=DEV)
    mark[0, 83:, 1, 5] = True
    assert not torch.isfinite(got[0, 83:90, 1, 5]).any()
    f32 = (4 * 150 + 32 + 64) * R.U32 + (U[dtype] if dtype is BF16 else 0.0)
    keep = ~mark.cpu().numpy()
    R.within(torch.where(mark, 0.0, got), np.where(keep, y, 0.0),
             U[dtype] * np.abs(y) + f32 * size, "finite rows")
    assert not torch.isfinite(layer.state[0, 1, 5]).any()
    S[0, 1, 5] = 0.0
    layer.state[0, 1, 5] = 0.0
    R.within(layer.state, S, (4 * 150 + 96) * R.U32 * M + 1e-300, "finite states")


# ------------------------------------------------------------ the mixer


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_mixer_is_its_layers(dtype):
    """The mixer's three layers against the plain forms run one after the other
    on the rounded values between them; steps against the clip."""
    B, T, H, P, G, N, K = 2, 70, 4, 32, 2, 32, 4
    case = (B, T, H, P, G, N, dtype, "full", True, True)
    g = gen(51)
    v, _ = scan_inputs(case, 51)
    inner, shared = H * P, G * N
    u = randn(g, B, T, 2 * inner + 2 * shared + H, scale=0.7, dtype=dtype)
    w = randn(g, inner + 2 * shared, K, scale=0.5, dtype=dtype)
    nw = randn(g, inner)
    n = torch.tensor([T, 33], dtype=torch.int32)
    conv = coinf.CoShortConv(w.to(DEV), batch=B)
    scan = scan_layer(case, v, None)
    mixer = coinf.Mixer(conv, scan, coinf.CoNorm(nw.to(DEV), gate="before"))
    assert mixer.width == u.shape[-1]
    got = mixer.forward(u.to(DEV), n.to(DEV))
    z, xbc, dt = u.split((inner, inner + 2 * shared, H), -1)
    y1, s1, _ = R.shortconv(R.np64(xbc), R.np64(w), None, None, n, "silu")
    mid = conv.forward(xbc.to(DEV), n.to(DEV))
    R.within(mid, y1, U[dtype] * np.abs(y1) + (K + 9) * R.U32 * s1, "mixer conv")
    x, b, c = (t.cpu() for t in mid.split((inner, shared, shared), -1))
    parts = dict(v, x=x.unflatten(-1, (H, P)), dt=dt, b=b.unflatten(-1, (G, N)),
                 c=c.unflatten(-1, (G, N)))
    y = scan.forward(*(parts[k].to(DEV) for k in ("x", "dt", "b", "c")), n.to(DEV))
    y2, s2, _, _ = scan_ref(case, parts, None, n)
    f32 = (4 * T + N + 64) * R.U32 + (U[dtype] if dtype is BF16 else 0.0)
    R.within(y, y2, U[dtype] * np.abs(y2) + f32 * s2, "mixer scan")
    rows = y.flatten(2).reshape(-1, inner)
    want, _ = R.norm(R.np64(rows), R.np64(z.reshape(-1, inner)), None, R.np64(nw), None, 1, 1e-5,
                     "before", None)
    R.within(got.reshape(-1, inner), want, (U[dtype] + 56 * R.U32) * np.abs(want), "mixer norm")
    # the same tokens as a piece and single steps
    ud, keep = u.to(DEV), got.float()
    one = [mixer.forward_steps(ud[:, :40])]
    one += [mixer.forward_step(ud[:, t])[:, None] for t in range(40, T)]
    both = torch.cat(one, 1).float()
    # one rounding of the scan's factors and one of its output each, in the norm's scale
    assert R.relative(both[0], R.np64(keep[0])) <= (4 * U[BF16] if dtype is BF16 else 1e-5)
    with pytest.raises(ValueError):
        coinf.Mixer(conv, scan, coinf.CoNorm(nw.to(DEV)))
    with pytest.raises(ValueError):
        coinf.Mixer(conv, scan, coinf.CoNorm(dim=inner + 1, gate="before"))


def test_example_streams_equal_clips():
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "stream_tokens.py")
    spec = importlib.util.spec_from_file_location("stream_tokens", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    assert mod.main(longest=130, tokens=6) < 0.03


# ------------------------------------------------------------ places that go wrong


@pytest.mark.parametrize("T", [4, 150])
@pytest.mark.parametrize("which", ["dt", "b", "c"])
def test_scan_nonfinite_inputs_reach_nothing_before_them(which, T):
    for dtype in (F32, BF16):
        case = (2, T, 2, 32, 1, 32, dtype, "full", True, True)
        v, _ = scan_inputs(case, 42)
        s = T * 2 // 3
        y, size, _, _ = scan_ref(case, v, v["state"], None)
        v[which][1, s] = float("nan")
        layer = scan_layer(case, v, v["state"])
        got = layer.forward_steps(*(v[k].to(DEV) for k in ("x", "dt", "b", "c")))
        assert torch.isnan(got[1, s]).all()
        if which != "c":
            assert torch.isnan(got[1, -1]).all() and torch.isnan(layer.state[1]).all()
        f32 = (4 * T + 96) * R.U32 + (U[dtype] if dtype is BF16 else 0.0)
        bound = U[dtype] * np.abs(y) + f32 * size
        R.within(got[0], y[0], bound[0], f"other stream {which}")
        R.within(got[1, :s], y[1, :s], bound[1, :s], f"before {which}")


def test_lengths_out_of_range_are_all_or_none():
    case = (3, 70, 2, 32, 1, 32, BF16, "full", True, True)
    v, _ = scan_inputs(case, 43)
    n, good = torch.tensor([-5, 71, 1 << 30]), torch.tensor([0, 70, 70])
    n, good = (t.to(torch.int32).to(DEV) for t in (n, good))
    d = [v[k].to(DEV) for k in ("x", "dt", "b", "c")]
    layer = scan_layer(case, v, None)
    assert torch.equal(layer.forward(*d, n), layer.forward(*d, good))
    conv = coinf.CoShortConv(torch.ones(64, 4, dtype=BF16, device=DEV), batch=3)
    x = d[0].flatten(2)
    assert torch.equal(conv.forward(x, n), conv.forward(x, good))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_without_workspace(dtype):
    """The C ABI without a workspace runs the call token by token, as accurate."""
    import ctypes

    case = (2, 90, 4, 32, 1, 32, dtype, "full", True, True)
    v, _ = scan_inputs(case, 44)
    layer = scan_layer(case, v, v["state"])
    d = {k: v[k].to(DEV) for k in ("x", "dt", "b", "c")}
    assert layer.workspace_bytes(90) > 0
    y = torch.empty_like(d["x"])
    parts = [coinf.Tokens(t.data_ptr(), t.stride(0), t.stride(1))
             for t in (d["x"], d["dt"], d["b"], d["c"], y)]
    for ws, nws in ((None, 0), (layer.state.data_ptr(), 16)):
        layer.state.copy_(v["state"])
        call = coinf.ScanCall(layer.A.data_ptr(), layer.D.data_ptr(), layer.dt_bias.data_ptr(),
                              *parts, None, layer.state.data_ptr(), ws, nws, 90, 1)
        st = coinf.co_scan_forward_steps(ctypes.byref(layer.desc), ctypes.byref(call),
                                         torch.cuda.current_stream().cuda_stream)
        assert st == coinf.CO_OK
        check_scan(case, y, layer.state, scan_ref(case, v, v["state"], None), "no workspace")


def far(t, apart):
    """t (2, T, ...) on the device with its two streams `apart` elements apart."""
    n = t[0].numel()
    room = torch.empty(apart + n, dtype=t.dtype, device=DEV)
    out = room.as_strided(t.shape, (apart,) + t.stride()[1:])
    out.copy_(t)
    return out


def test_offsets_past_32_bits():
    """Streams more than 2^32 elements apart, in and out."""
    apart = (1 << 32) + 64
    case = (2, 70, 2, 32, 1, 32, BF16, "full", True, True)
    v, _ = scan_inputs(case, 45)
    layer = scan_layer(case, v, v["state"])
    d = {k: v[k].to(DEV) for k in ("x", "dt", "b", "c")}
    want = layer.forward(*d.values())
    x, out = far(v["x"], apart), far(torch.zeros_like(v["x"]), apart)
    for T in (70, 3):
        got = layer.forward(x[:, :T], *(d[k][:, :T] for k in ("dt", "b", "c")), out=out[:, :T])
        keep = want if T == 70 else layer.forward(*(t[:, :3] for t in d.values()))
        assert torch.equal(got, keep)
    conv = coinf.CoShortConv(torch.randn(64, 4, dtype=BF16, device=DEV), batch=2)
    u, o = x.flatten(2), out.flatten(2)
    assert torch.equal(conv.forward(u, out=o), conv.forward(d["x"].flatten(2)))
    norm = coinf.CoNorm(dim=64, gate="before")
    assert torch.equal(norm.forward(u, gate=u, out=o),
                       norm.forward(d["x"].flatten(2), gate=d["x"].flatten(2)))


def test_scan_tokens_far_apart():
    """Tokens 2^22 elements apart and more: a chunk's offsets take more than 31 bits."""
    case = (1, 70, 2, 32, 1, 32, F32, "full", True, True)
    v, _ = scan_inputs(case, 46)
    layer = scan_layer(case, v, None)
    d = {k: v[k].to(DEV) for k in ("x", "dt", "b", "c")}
    wide = torch.empty(70, (1 << 24) + 64, device=DEV)           # 4.7 GB
    x = wide[:, :64].unflatten(-1, (2, 32))[None]
    x.copy_(d["x"])
    got = layer.forward(x, *(d[k] for k in ("dt", "b", "c")))
    y, size, _, _ = scan_ref(case, v, None, None)
    R.within(got, y, U[F32] * np.abs(y) + (4 * 70 + 96) * R.U32 * size, "far tokens")


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_single_token_forms(dtype):
    """forward_step is forward_steps of one token, bit for bit: slices, an out
    tensor, streams without a token, no update; and its refusals."""
    g = gen(61)
    B, H, P, G, N = 3, 4, 16, 2, 20
    n = torch.tensor([1, 0, 1], dtype=torch.int32, device=DEV)
    wide = randn(g, B, H * P + 2 * G * N + H, dtype=dtype).to(DEV)
    x, b, c, dt = wide.split((H * P, G * N, G * N, H), -1)
    x, b, c = x.view(B, H, P), b.view(B, G, N), c.view(B, G, N)
    w = randn(g, H * P, 3, dtype=dtype).to(DEV)
    xc = wide[:, 5:5 + H * P]
    convs = [coinf.CoShortConv(w, batch=B) for _ in range(2)]
    scans = [coinf.CoScan(-torch.ones(H, device=DEV), batch=B, head_dim=P, state_size=N, groups=G,
                          dtype=dtype) for _ in range(2)]
    for lengths, update in ((None, True), (n, True), (None, False), (n, False)):
        out = torch.full((B, 2 * H * P), 7., dtype=dtype, device=DEV)
        want = convs[0].forward_steps(xc[:, None], lengths, update)[:, 0]
        got = convs[1].forward_step(xc, lengths, update, out=out[:, 3:3 + H * P])
        assert torch.equal(got, want) and torch.equal(out[:, 3:3 + H * P], want)
        assert (out[:, :3] == 7).all() and (out[:, 3 + H * P:] == 7).all()
        assert torch.equal(convs[0].state, convs[1].state)
        want = scans[0].forward_steps(x[:, None], dt[:, None], b[:, None], c[:, None], lengths,
                                      update)[:, 0]
        got = scans[1].forward_step(x, dt, b, c, lengths, update)
        assert torch.equal(got, want) and torch.equal(scans[0].state, scans[1].state)
        out = torch.full((B, 2, H, P), 7., dtype=dtype, device=DEV)
        scans[1].forward_step(x, dt, b, c, lengths, False, out=out[:, 1])
        assert (out[:, 0] == 7).all()
    conv, scan = convs[0], scans[0]
    for f in (lambda: conv.forward_step(xc[:, None]), lambda: conv.forward_steps(xc),
              lambda: conv.forward(xc), lambda: conv.forward_step(xc[:2]),
              lambda: conv.forward_step(xc, out=torch.empty_like(xc)[:, None]),
              lambda: scan.forward_step(x[:, None], dt, b, c),
              lambda: scan.forward_step(x, dt[:, None], b, c),
              lambda: scan.forward_step(x, dt, b[:, None], c),
              lambda: scan.forward_step(x, dt, b, c[:, :1]),
              lambda: scan.forward_steps(x, dt, b, c),
              lambda: scan.forward_step(x, dt, b, c, out=torch.empty_like(x)[:, None])):
        with pytest.raises(ValueError):
            f()
    # a refused call leaves the next one's arguments checked anew
    assert torch.equal(conv.forward_step(xc, update_state=False),
                       convs[1].forward_step(xc, update_state=False))
