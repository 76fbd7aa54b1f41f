"""Without a GPU: what the tables of spo_grad_norm and spo_adamw_update hold on to."""

import gc
import weakref

import numpy as np
import pytest

from paper_2509_13232_b200 import binding as B


class Held:
    """Tensors whose memory can be watched."""

    def __init__(self, torch):
        self.torch, self.memory = torch, []

    def __call__(self, n=1000, dtype=np.float32):
        x = np.zeros(n, dtype)
        self.memory.append(weakref.ref(x))
        return self.torch.from_numpy(x)

    def alive(self):
        gc.collect()
        return [x() is not None for x in self.memory]


@pytest.fixture
def held(monkeypatch):
    import torch
    monkeypatch.setattr(B, "_one_device", lambda torch, tensors: 0)
    return Held(torch)


def test_memory_of_a_list_stays_while_the_list_does(held):
    """Tensors that are given other memory (p.data = ..., p.set_(...)) leave the list's to the list: the addresses in its table are not
    given back while a step may still use them."""
    import torch
    w, g, m, v = held(), held(), held(dtype=np.int8), held(dtype=np.uint8)
    ms, vs = held(4), held(4)
    table = B.adamw_list([w], [g], [m], [v], [ms], [vs])
    for t in (w, g, m):
        t.data = torch.empty(1000, dtype=t.dtype)
    for t in (v, ms, vs):
        t.set_(torch.empty(1000, dtype=t.dtype))
    assert all(held.alive())
    del table
    assert not any(held.alive())


def test_memory_of_gradients_stays_with_their_list(held):
    import torch
    g = [held(), held(7)]
    grads = B.grad_list(g)
    g[0].data = torch.empty(5)
    del g
    assert held.alive() == [True, True]
    del grads
    assert held.alive() == [False, False]
