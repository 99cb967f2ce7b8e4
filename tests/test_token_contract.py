"""What the token layers promise, as far as the host shows it.  No GPU."""
import ctypes

import pytest
import torch

from paper_2204_03418_amd import coinf as C
from test_token_abi import P, norm, ref, scan


def test_norm_lengths_arguments():
    t = [C.Tokens(*v) if v else C.Tokens() for v in ((P, 48, 16), None, None, (P, 48, 16), None)]
    call = C.NormCall(*t, P, None)
    run = lambda d, n: C.co_norm_forward_lengths(ref(d), ref(call), n, None)  # noqa: E731
    assert run(norm(batch=0), None) == C.CO_OK and run(norm(tokens=0), P) == C.CO_OK
    assert run(norm(), P + 2) == C.CO_EINVAL                    # not an int32's address
    assert run(norm(eps=-1.0), P) == C.CO_EINVAL
    assert C.co_norm_forward_lengths(ref(norm()), None, P, None) == C.CO_EINVAL
    assert ctypes.sizeof(C.NormCall) == 5 * 24 + 16             # as co_norm_forward's callers have it


class OnDevice:
    """The part of a device tensor that the binding looks at, on any device."""

    def __init__(self, index, shape, dtype=torch.float32):
        self.device, self.shape, self.dtype = torch.device("cuda", index), torch.Size(shape), dtype
        self.is_cuda = True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self, axis=None):
        st = [1]
        for n in reversed(self.shape[1:]):
            st.insert(0, st[0] * n)
        return tuple(st) if axis is None else st[axis]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P


def test_tensors_of_another_gpu_are_refused():
    here, shape = torch.device("cuda", 0), torch.Size((2, 5, 8))
    into = C.Tokens()
    C._tokens(OnDevice(0, shape), torch.float32, shape, "x", into, here)
    assert (into.batch_stride, into.token_stride) == (40, 8)
    with pytest.raises(ValueError, match="cuda:1"):
        C._tokens(OnDevice(1, shape), torch.float32, shape, "x", into, here)
    n = (2,), torch.int32
    assert C._lengths(OnDevice(0, *n), 2, here) == P
    with pytest.raises(ValueError, match="cuda:1"):
        C._lengths(OnDevice(1, *n), 2, here)
    norm_layer = C.CoNorm(dim=8)
    norm_layer._rows(OnDevice(1, shape), torch.float32, shape, 5, "x", into, torch.device("cuda", 1))
    with pytest.raises(ValueError, match="cuda:1"):
        norm_layer._rows(OnDevice(1, shape), torch.float32, shape, 5, "gate", into, here)


@pytest.mark.parametrize("big", [
    dict(batch=1, heads=1 << 20, head_dim=1, state_size=1, groups=1),
    dict(batch=1, heads=1 << 17, head_dim=4, state_size=16, groups=1 << 17),
    dict(batch=1 << 12, heads=1 << 13, head_dim=1, state_size=1, groups=1 << 13)], ids=str)
def test_scan_workspace_of_calls_too_wide_for_chunks(big):
    """What a launch of the chunked form cannot hold runs token by token, which
    wants no workspace."""
    n = C.i64(-1)
    assert C.co_scan_workspace_bytes(ref(scan(**big)), 1000, ref(n)) == C.CO_OK and n.value == 0
    small = dict(big, batch=1, heads=16, groups=min(big["groups"], 16))
    assert C.co_scan_workspace_bytes(ref(scan(**small)), 1000, ref(n)) == C.CO_OK and n.value > 0


def test_norm_in_place_means_the_same_places():
    """An output at an input's address but with other strides or another element
    size would be written over rows that are still to be read."""
    def call(d, x=(P, 48, 16), gate=None, residual=None, y=(8 * P, 48, 16), out=None):
        t = [C.Tokens(*v) if v else C.Tokens() for v in (x, gate, residual, y, out)]
        return C.co_norm_forward(ref(d), ref(C.NormCall(*t, None, None)), None)

    sizes = dict(batch=2, tokens=3, dim=16)
    turned = (P, 16, 32)                                        # streams beside each other
    assert call(norm(**sizes), y=turned) == C.CO_EINVAL
    assert call(norm(**sizes, gate=1), gate=(3 * P, 48, 16), y=(3 * P, 96, 16)) == C.CO_EINVAL
    both = dict(sizes, residual=1, dtype=C.CO_BF16, residual_dtype=C.CO_F32)
    assert call(norm(**both), residual=(4 * P, 48, 16), out=(P, 48, 16)) == C.CO_EINVAL
    assert call(norm(**both), residual=(4 * P, 48, 16), y=(4 * P, 48, 16),
                out=(5 * P, 48, 16)) == C.CO_EINVAL
    assert call(norm(**sizes, residual=1), residual=(4 * P, 48, 16), y=(5 * P, 48, 16),
                out=(5 * P, 48, 16)) == C.CO_EINVAL             # both outputs in one place
