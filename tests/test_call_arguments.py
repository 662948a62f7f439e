"""What dopr_prefix_attn and dopr_gather_prefix take as arguments, on the CPU: a
store that was closed, which the library refuses once the arguments have become
the C call's."""
import ctypes

import numpy as np
import pytest
import torch


def _D():
    import paper_2609_03311_amd as D
    D.lib()
    return D


class Closed:
    handle, n_kv_heads, head_dim = None, 2, 128


class Stream:
    cuda_stream = 0


class Memory:
    """What a call asks of a tensor, and no torch tensor."""

    def __init__(self, *shape):
        self.shape = shape

    def data_ptr(self):
        return 256

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return 2


def _attention(layer=0, **more):
    ids = torch.zeros(1, dtype=torch.int32)
    cu = torch.tensor([0, 3], dtype=torch.int32)
    x = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    args = dict(doc_ids=ids, cu_seqlens=cu, q=x, k=x, v=x, q_norm_w=None,
                k_norm_w=None, out=x, workspace=torch.zeros(256), max_tokens=3,
                stream=Stream())
    args.update(more)
    return lambda D: D.dopr_prefix_attn(Closed(), layer, **args)


def _gather(layer=0, **more):
    args = dict(doc_ids=torch.zeros(1, dtype=torch.int32),
                out_cu_slots=torch.tensor([0, 3]), k_out=torch.zeros(3),
                v_out=torch.zeros(3), stream=Stream())
    args.update(more)
    return lambda D: D.dopr_gather_prefix(Closed(), layer, **args)


class Other(Stream):
    cuda_stream = ctypes.c_void_p(16)


TAKEN = {
    "as usual": _attention(),
    "whole numbers of numpy": _attention(np.int32(0), max_tokens=np.int64(3),
                                         total_tokens=np.int64(3)),
    "numbers in another form": _attention(max_tokens=3.0, rms_eps=1,
                                          rope_theta=np.float32(1e4),
                                          kernel_variant="8",
                                          softmax_scale="0.1"),
    "memory that is no tensor": _attention(
        doc_ids=Memory(1), cu_seqlens=Memory(2), q=Memory(3, 4, 128),
        k=Memory(3, 2, 128), v=Memory(3, 2, 128), out=Memory(3, 4, 128),
        workspace=Memory(256), lse=Memory(3, 4)),
    "handles of ctypes": _attention(timing=(ctypes.c_void_p(16),
                                            ctypes.c_void_p(32)),
                                    stream=Other()),
    "events": _attention(timing=(16, 32)),
    "read back": _gather(),
    "read back into memory that is no tensor": _gather(
        np.int64(0), doc_ids=Memory(1), out_cu_slots=Memory(2),
        k_out=Memory(3), v_out=Memory(3), stream=Other()),
}


@pytest.mark.parametrize("what", list(TAKEN))
def test_taken(what):
    D = _D()
    with pytest.raises(D.DoprError, match="store is NULL"):
        TAKEN[what](D)


REFUSED = {
    "a part of a layer": (_attention(1.7), ctypes.ArgumentError),
    "a layer in text": (_attention("0"), ctypes.ArgumentError),
    "no layer": (_attention(None), ctypes.ArgumentError),
    "no documents": (_attention(doc_ids=None), AttributeError),
    "no q, no count": (_attention(q=None), AttributeError),
    "no kv heads in q": (_attention(q=torch.zeros(3)), IndexError),
    "an address for a tensor": (_attention(out=256), AttributeError),
    "an event as a fraction": (_attention(timing=(1.5, 2.5)), TypeError),
    "no number": (_attention(rms_eps="x"), ValueError),
    "a part of a layer to read": (_gather(0.5), ctypes.ArgumentError),
    "a layer to read in text": (_gather("1"), ctypes.ArgumentError),
    "a list of documents": (_gather(doc_ids=[0]), AttributeError),
    "an address to read to": (_gather(k_out=256), AttributeError),
}


@pytest.mark.parametrize("what", list(REFUSED))
def test_refused(what):
    D = _D()
    call, error = REFUSED[what]
    with pytest.raises(error):
        call(D)
