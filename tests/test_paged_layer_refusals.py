"""What the decoder layer over pages refuses of its layer on the host: before its first launch, so that a refused step has
written no row to the pages."""
import ctypes

import pytest

from test_kv_refusals import OK, SHAPE, UNSUPPORTED, L, cache  # noqa: F401


def step(L, h, kv, hd=64, d=512, n_pos=8, m=2):  # noqa: F811
    from paper_2606_04238_gb300 import wq
    q = lambda n, k, bits: wq._QWeight(256, 512, n, k, 128, bits)  # noqa: E731
    mlp = wq._MLPLayer(q(1024, d, 2), q(1024, d, 2), q(d, 1024, 4), None, None, None, 0, 0.0)
    layer = wq._DecoderLayer(q((h + 2 * kv) * hd, d, 4), q(d, h * hd, 4), mlp, h, kv, hd, 1e6)
    pool = cache(batch=8, max_len=32, n_kv=kv, head_dim=hd)
    return L.wq_decoder_paged_forward(256, m, m, 1, 256, 512, 256, 512, ctypes.byref(layer), None, None, pool, 256, 4, 512, n_pos, 0, 256,
                                      256, 1 << 40, None)


@pytest.mark.parametrize("h,kv", [(34, 2), (20, 1), (6, 4)])
def test_query_heads_a_kv_head(L, h, kv):  # noqa: F811
    assert step(L, h, kv) == UNSUPPORTED and b"query heads" in L.wq_last_error()
    assert step(L, h, kv, m=0) == UNSUPPORTED


def test_a_table_without_positions(L):  # noqa: F811
    assert step(L, 8, 2, n_pos=0) == SHAPE and b"table" in L.wq_last_error()


def test_nothing_to_do(L):  # noqa: F811
    assert step(L, 8, 2, m=0) == OK and step(L, 8, 2, m=0, n_pos=0) == OK
