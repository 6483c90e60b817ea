"""What the binding of the drafted calls does by itself, without a GPU."""
import gc
import weakref

import torch

from helpers import load_binding


def test_rows_keep_their_tensors():
    """The address of a temporary is not another tensor's by the time of the call."""
    cqa = load_binding()
    x = torch.zeros((2, 3, 128))
    st = (384, 128, 128)
    made = x.transpose(0, 1).contiguous()
    ref, at = weakref.ref(made), made.data_ptr()
    rows = [cqa.RotaryRows(made, x, 3, st, st)]
    del made
    gc.collect()
    assert ref() is not None and rows[0].in_dev == at and rows[0].out_dev == x.data_ptr()
    del rows
    gc.collect()
    assert ref() is None
    assert cqa.RotaryRows(4096, None, 1, st, st).out_dev is None
