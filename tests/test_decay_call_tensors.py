"""What the Python calls of decayed linear attention and draft verification look at before they pass an address on (no GPU: tensors that only say
that they are on one, and a host-only plan, at which the library stops)."""
import numpy as np
import pytest
import torch

import paper_2608_30386_b200 as dasc
from paper_2608_30386_b200 import binding

P = 0x1000  # an aligned address that is never followed


class Tensor:
    """Says what a tensor on the current device would."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=0, contiguous=True):
        self.shape, self.dtype, self.device_index, self.contiguous = shape, dtype, device, contiguous

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return self.dtype.itemsize

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return P


class Stream:
    cuda_stream = 0


def attn(**changes):
    plan = dasc.dasc_plan(dasc.GDN, 1, 2, 2, 128, 128, np.zeros(2, np.float32), np.zeros(2, np.float32), device=-1)
    x = lambda: Tensor(1, 4, 2, 128)  # noqa: E731
    i = lambda n: Tensor(n, dtype=torch.int32)  # noqa: E731
    a = dict(state=Tensor(4, 32768, dtype=torch.float32), layer_stride=32768, req_stride=32768, req_idx=i(4), q=x(), k=x(), v=x(),
             g=Tensor(1, 4, 2, dtype=torch.float32), cu_seqlens=i(5), total_tokens=4, max_seqlen=4, o=x(), workspace=None, stream=Stream())
    dasc.dasc_decay_attn(plan, **{**a, **changes})


def test_a_call_with_nothing_wrong_reaches_the_library():
    for changes in ({}, dict(state=P, g=P, seq_used=P), dict(workspace=Tensor(4096, dtype=torch.uint8))):
        with pytest.raises(dasc.DascError) as e:
            attn(**changes)
        assert e.value.status == binding.ERR_INVALID_ARG  # a plan without a device


@pytest.mark.parametrize("name", ["q", "k", "v", "o"])
def test_an_address_does_not_say_of_which_type_its_values_are(name):
    with pytest.raises(TypeError, match=f"^{name} "):
        attn(**{name: P})


@pytest.mark.parametrize("bad, message", [(dict(device=-1), "device"), (dict(device=1), "device"), (dict(contiguous=False), "contiguous")])
def test_a_workspace_is_looked_at_like_every_other_tensor(bad, message):
    """On the host, on another device, or a strided view, whose count of values says nothing about how far it reaches."""
    with pytest.raises(ValueError, match=f"^workspace .*{message}"):
        attn(workspace=Tensor(4096, dtype=torch.uint8, **bad))
