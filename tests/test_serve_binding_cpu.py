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


def test_tensors_in_host_memory():
    """The kernels would follow a pointer into the host's memory: every tensor of every call is looked at."""
    f32, u8 = torch.zeros(2, 4, 32), torch.zeros(4, 16, dtype=torch.uint8)
    a = append_args()
    where = [a[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale", "block_table", "start", "kv_len")]
    for call in (lambda: C.crvq_kv_append(**a), lambda: C.crvq_kv_read(a["k"], None, *where, 2),
                 lambda: C.crvq_kv_attention(f32, f32.clone(), *where, 2, 2),
                 lambda: C.crvq_w4_quantize(torch.zeros(4, 32), u8, torch.zeros(4, 1), 32),
                 lambda: C.crvq_w4_dequant(u8, torch.zeros(4, 1), 32, torch.zeros(4, 32)),
                 lambda: C.crvq_w4_gemv(u8, torch.zeros(4, 1), 32, torch.zeros(1, 32), torch.zeros(1, 4))):
        with pytest.raises(ValueError, match="host memory"):
            call()


class OnGpu(torch.Tensor):
    """A tensor that says it is on the GPU, so that the one left on the host can be found without one."""
    is_cuda = True


@pytest.mark.parametrize("host", ["k", "v", "q", "q_out", "k_cache", "v_cache", "k_scale", "v_scale", "block_table", "start", "kv_len",
                                  "cos", "sin", "positions"])
def test_one_tensor_in_host_memory(host):
    a = append_args(q=torch.zeros(2, 4, 32), q_out=torch.zeros(2, 4, 32), cos=torch.zeros(4, 16), sin=torch.zeros(4, 16),
                    positions=torch.zeros(2, dtype=torch.int32))
    a = {n: t.as_subclass(OnGpu) if n != host and isinstance(t, torch.Tensor) else t for n, t in a.items()}
    with pytest.raises(ValueError, match="host memory"):
        C.crvq_kv_append(**a)
