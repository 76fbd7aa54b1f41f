"""What the binding refuses of a call with alternatives, rather than leave a tensor of it unwritten."""

import pytest

pytestmark = pytest.mark.gpu


def test_alternatives_come_as_a_pair():
    import torch
    from paper_2509_13232_b200 import binding as B
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    H, W = f(4, 64).bfloat16(), f(10, 64).bfloat16()
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    ids = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    call = lambda i, t: B.spo_logprobs(H, W, None, None, None, f(4), None, i, t, ws, None)  # noqa: E731
    call(ids(4, 2), f(4, 2))
    call(ids(4, 0), f(4, 0))
    call(None, None)
    for i, t in ((None, f(4, 2)), (ids(4, 2), None), (ids(4, 0), f(4, 2)), (ids(4, 2), f(4, 3)), (ids(4), f(4)), (ids(3, 2), f(3, 2)),
                 (ids(()), f(())), (ids(3, 0), f(3, 0)), ([1, 2], f(4, 2))):
        with pytest.raises((TypeError, ValueError)):
            call(i, t)
    torch.cuda.synchronize()
