"""CPU-only: calls that no launch has threads for are refused (a launch of 2^32 threads or more is cut short without an error)."""
import pytest

from paper_2604_09975_amd import binding as B
from paper_2604_09975_amd import clear as K
from tests.test_clear_abi import P, grad, last

PAGES = dict(k=P, v=2 * P, ks0=2048, ks1=1024, ks2=64, vs0=2048, vs1=1024, vs2=64)
PACKED = dict(k=P, v=2 * P, kz=3 * P, vz=4 * P, ks0=2048, ks1=1024, ks2=64, vs0=2048, vs1=1024, vs2=64, kz0=64, kz1=32, kz2=2, vz0=64, vz1=32, vz2=2)
BATCH = dict(q_start=5 * P, kv_len=6 * P, table=7 * P, ts=1)
# (far apart: what is asked of the arrays' places comes later)
CALL = dict(q=1 << 50, out=1 << 51, lse=0, work=0, bytes=0, q0=256, q1=64, o0=256, o1=64, heads=4, window=0, flags=1, scale=0.125)


def plain(dtype, n_tokens, n_seq):
    return K._ATTEND(*PAGES.values(), 10, 16, 2, 64, dtype, 0, *BATCH.values(), n_seq, n_tokens, 1, 0, *CALL.values())


def packed(dtype, n_tokens, n_seq):
    return K._PACKED_ATTEND(*PACKED.values(), 10, 16, 2, 64, 16, dtype, *BATCH.values(), n_seq, n_tokens, 1, 0, *CALL.values())


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("name,pack", [("attend", plain), ("packed_attend", packed)])
def test_attention_of_more_blocks_than_a_launch_has(name, pack, dtype):
    """Single tokens of 2^23 sequences: a block of 256 threads for each of two kv heads."""
    n = 1 << 23
    args = pack(dtype, n, n)
    assert getattr(B.lib, f"ckks_clear_{name}")(args, None) == -1 and "tokens" in last() and name in last()
    assert getattr(B.lib, f"ckks_clear_{name}_work_bytes")(args) == 0


def test_gradients_of_more_weights_than_a_launch_has_threads_for():
    work = B.lib.ckks_clear_layer_norm_grad_work_bytes(1, 1 << 28, 0)
    far = dict(dy=1 << 50, x=2 << 50, w=0, dx=0, dw=3 << 50, db=4 << 50, work=5 << 50)
    assert grad(rows=1, cols=1 << 28, bytes=work, **far) == -1 and "one launch" in last()
