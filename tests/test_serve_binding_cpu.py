"""CPU-only: what the binding of the quantized attention block's calls refuses before the library sees it."""
import pytest
import torch

from paper_2412_09282_amd import crvq as C


def append_args(**kw):
    i32 = dict(dtype=torch.int32)
    a = dict(k=torch.zeros(2, 2, 32), v=torch.zeros(2, 2, 32), k_cache=torch.zeros(1, 2, 16, 32, dtype=torch.int8),
             v_cache=torch.zeros(1, 2, 32, 16, dtype=torch.int8), k_scale=torch.zeros(1, 2), v_scale=torch.zeros(1, 2),
             block_table=torch.zeros(1, 1, **i32), start=torch.tensor([0, 2], **i32), kv_len=torch.tensor([2], **i32), max_new=2)
    a.update(kw)
    return a


def test_append_arguments_that_go_together():
    angles, q = torch.zeros(4, 16), torch.zeros(2, 4, 32)
    for bad in (dict(sin=angles), dict(cos=angles), dict(q=q), dict(q_out=q), dict(cos=angles, sin=angles, q_out=q)):
        with pytest.raises(ValueError, match="go together"):
            C.crvq_kv_append(**append_args(**bad))
