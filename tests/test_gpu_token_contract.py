"""What the token layers promise beyond their formulas: how exact bfloat16 is,
what lies past a stream's length, layers in chains, and which arguments they
refuse.

Bounds as in test_gpu_tokens.py: `size` is the sum of an output's magnitudes, u
a dtype's unit roundoff.
"""
import numpy as np
import pytest
import torch

import token_ref as R
from paper_2204_03418_amd import coinf
from test_gpu_tokens import BF16, DEV, U, scan_inputs, scan_layer, scan_ref

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------ bfloat16


@pytest.mark.parametrize("case", [
    # B, T, H, P, G, N, dtype, lengths, softplus, D
    (1, 64, 2, 32, 1, 32, BF16, "full", True, True),
    (2, 150, 4, 64, 2, 64, BF16, "ragged", True, True),
    (2, 90, 4, 64, 1, 128, BF16, "full", False, False),
    (1, 130, 3, 40, 1, 20, BF16, "full", True, True),
    (1, 100, 2, 64, 1, 256, BF16, "full", True, True),
    (1, 900, 4, 64, 2, 128, BF16, "full", True, True),
], ids=str)
def test_scan_bfloat16_is_rounded_once(case):
    """A prompt's outputs in bfloat16 are float32 sums rounded once, also where
    the sum cancels: the float32 factors of its products keep 16 bits at least
    (two bfloat16 terms leave u^2 of a value, u = 2^-8).  And they are those of
    single tokens, but for that and the two roundings."""
    T, N = case[1], case[5]
    v, n = scan_inputs(case, 71)
    layer = scan_layer(case, v, v["state"])
    d = [v[k].to(DEV) for k in ("x", "dt", "b", "c")]
    nd = None if n is None else n.to(DEV)
    assert layer.workspace_bytes(T) > 0                         # the chunks take the call
    got = layer.forward_steps(*d, nd, update_state=False)
    y, size, _, _ = scan_ref(case, v, v["state"], n)
    f32 = (4 * T + N + 64) * R.U32
    keep = U[BF16] ** 2 + f32
    R.within(got, y, U[BF16] * np.abs(y) + keep * size, f"bfloat16 {case}")
    steps = []
    for t in range(T):
        on = None if n is None else (n > t).to(torch.int32).to(DEV)
        steps.append(layer.forward_step(*(a[:, t] for a in d), on))
    # each value within its own bound of the sum; what is rounded is no larger than the
    # sum and the error before
    most = 2 * U[BF16] * (np.abs(y) + keep * size) + (keep + f32) * size
    R.within(got, R.np64(torch.stack(steps, 1)), most, f"bfloat16 steps {case}")


# ------------------------------------------------------------ pieces shorter than the state


@pytest.mark.parametrize("K", [4, 5, 6, 8])
@pytest.mark.parametrize("T", [3, 6, 8, 13])
def test_drafted_pieces_are_single_tokens(K, T):
    """A few drafted tokens of many streams, twice, against single tokens bit for
    bit: outputs and the state, which a piece reads and writes in one launch."""
    g = torch.Generator().manual_seed(81)
    B, C = 32, 1088
    x = torch.randn(B, 2 * T, C, generator=g).to(BF16).to(DEV)
    w = torch.randn(C, K, generator=g).to(BF16).to(DEV)
    state = torch.randn(B, K - 1, C, generator=g).to(BF16).to(DEV)
    n = torch.randint(0, T + 1, (B,), generator=g).to(torch.int32)
    pieces, steps = (coinf.CoShortConv(w, batch=B, state=state.clone()) for _ in range(2))
    for part, lengths in ((x[:, :T], None), (x[:, T:], n)):
        nd = None if lengths is None else lengths.to(DEV)
        got = pieces.forward_steps(part, nd)
        want = torch.stack([steps.forward_step(
            part[:, t], None if lengths is None else (lengths > t).to(torch.int32).to(DEV))
            for t in range(T)], 1)
        assert torch.equal(got, want) and torch.equal(pieces.state, steps.state)


# ------------------------------------------------------------ past a stream's length


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
@pytest.mark.parametrize("wide", [True, False])
@pytest.mark.parametrize("which", ["x", "dt", "b", "c", "state"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_scan_past_lengths_is_zero_whatever_the_stream_holds(which, bad, wide, dtype):
    """Outputs past a stream's length are 0 also where its own tokens or its
    state are not finite, in one segment and in several, in pieces of 16 bytes
    and value by value."""
    for B, T, H in ((3, 150, 4), (3, 700, 2)):
        P, N = (32, 32) if wide else (33, 21)
        case = (B, T, H, P, 2, N, dtype, "full", True, True)
        v, _ = scan_inputs(case, 72)
        n = torch.tensor([T - 50, 41, 0], dtype=torch.int32)
        if which == "state":
            v["state"][:, 1, 3, 2] = bad
        else:
            v[which][0, T - 53], v[which][1, 3] = bad, bad
        layer = scan_layer(case, v, v["state"])
        assert layer.workspace_bytes(T) > 0
        got = layer.forward_steps(*(v[k].to(DEV) for k in ("x", "dt", "b", "c")), n.to(DEV))
        for i, k in enumerate(n.tolist()):
            assert (got[i, k:] == 0).all(), (which, i)
        assert not torch.isfinite(got[0, :T - 50]).all()
