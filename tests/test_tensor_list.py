"""A TensorList stands for the memory that its tensors had when it was made: it keeps that alive, and a call is refused once a tensor has other memory."""
import gc
import weakref

import numpy as np
import pytest
import torch

from paper_2510_24211_amd import binding as B
from test_table_binding import _gpu, _scd

F32 = torch.float32


class OnCard(torch.Tensor):
    """A tensor in host memory that says it is a GPU's: nothing here is launched."""
    is_cuda = True


def _card(*shape):
    return torch.ones(*shape).as_subclass(OnCard)


def _exchange(t):
    t.data = _card(2000)


def _set(t):
    t.set_(_card(2000).untyped_storage())


def _grow(t):
    t.resize_(1 << 20)


def _release(t):
    t.untyped_storage().resize_(0)


@pytest.mark.parametrize("change", [_exchange, _set, _grow, _release])
def test_calls_are_refused_once_a_tensor_has_other_memory(change):
    s, good, t = _scd(), _card(5), _card(2000)
    ts = B.TensorList([good, t])
    other = B.TensorList([_card(5), _card(2000)])
    change(t)
    norm, ws = _gpu(F32, 1), _gpu(torch.uint8, 1 << 20)
    for call in (lambda: s.gradient_norm(ts, norm, ws), lambda: s.clip_gradients(ts, other, 1.0, norm), lambda: s.clip_gradients(other, ts, 1.0, norm)):
        with pytest.raises(ValueError, match="tensor 1"):
            call()


def test_memory_lives_as_long_as_the_list(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)             # (a subclass would keep its memory by itself)
    memory = np.ones(2000, dtype=np.float32)
    t, alive = torch.from_numpy(memory), weakref.ref(memory)
    ts, address = B.TensorList([t]), t.data_ptr()
    del memory
    t.data = torch.ones(2000)
    gc.collect()
    assert alive() is not None and ts.array[0].d == address
    del ts
    gc.collect()
    assert alive() is None


def test_lists_of_what_has_no_elements_and_of_views():
    whole = _card(100)
    ts = B.TensorList([whole[3:3], whole[1:40], whole[40:]])
    ts.check("grads")
    assert [(x.n, x.d) for x in ts.array][1:] == [(39, whole.data_ptr() + 4), (60, whole.data_ptr() + 160)]
    B.TensorList([]).check("grads")
