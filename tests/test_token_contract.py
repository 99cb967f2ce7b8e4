"""What the token layers promise, as far as the host shows it.  No GPU."""
import ctypes

from paper_2204_03418_amd import coinf as C
from test_token_abi import P, norm, ref


def test_norm_lengths_arguments():
    t = [C.Tokens(*v) if v else C.Tokens() for v in ((P, 48, 16), None, None, (P, 48, 16), None)]
    call = C.NormCall(*t, P, None)
    run = lambda d, n: C.co_norm_forward_lengths(ref(d), ref(call), n, None)  # noqa: E731
    assert run(norm(batch=0), None) == C.CO_OK and run(norm(tokens=0), P) == C.CO_OK
    assert run(norm(), P + 2) == C.CO_EINVAL                    # not an int32's address
    assert run(norm(eps=-1.0), P) == C.CO_EINVAL
    assert C.co_norm_forward_lengths(ref(norm()), None, P, None) == C.CO_EINVAL
    assert ctypes.sizeof(C.NormCall) == 5 * 24 + 16             # as co_norm_forward's callers have it
