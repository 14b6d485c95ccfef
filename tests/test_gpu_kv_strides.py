"""wq_kv_append of tensors with a dimension of one, whose stride there addresses nothing and
may be any number."""
import pytest
import torch

from test_gpu_kv import _rows, _same, stored, wq  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("b,t,h", [(1, 5, 2), (3, 1, 2), (2, 6, 1), (1, 1, 1)])
def test_strides_of_dimensions_of_one(wq, dtype, b, t, h):
    hd = 64
    rows = _rows((b, t, h, hd), dtype, 1).cuda()
    given = list(rows.stride())
    for i, n in enumerate((b, t, h)):
        if n == 1:
            given[i] = 4099 + i
    odd = torch.as_strided(rows, rows.shape, given)
    start = torch.zeros(b, dtype=torch.int32, device="cuda")
    for bits in (16, 8):
        c = wq.kv_cache(b, h, t, hd, bits)
        wq.kv_append(c, odd, odd, start)
        k, v = wq.kv_read(c, start, t, dtype=torch.float32)
        assert _same(k, stored(rows, bits)[0]) and _same(v, stored(rows, bits)[0])
    two = torch.as_strided(torch.zeros(2 * 4099, dtype=dtype, device="cuda"), (2, 1, 1, hd), (4099, 1, 1, 1))
    with pytest.raises(wq.WQError) as e:
        wq.kv_append(wq.kv_cache(2, 1, 1, hd, 8), two, two, torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert e.value.status == -3
