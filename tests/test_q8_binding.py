"""What the Python binding of the 8-bit caches refuses before the C side sees it (no GPU needed: no call gets that far)."""
import pytest
import torch

from paper_2506_06266_b200 import binding as B, buildlib

BF, HALF, F32, F64 = torch.bfloat16, torch.float16, torch.float32, torch.float64


@pytest.fixture(autouse=True, scope="module")
def built():
    buildlib.build()


def t(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("q,out,lse", [
    (t(1, 4, 128, dtype=HALF), t(1, 4, 128), None), (t(1, 4, 128), t(1, 4, 128, dtype=F32), None),
    (t(1, 4, 256)[..., ::2], t(1, 4, 128), None), (t(1, 4, 128), t(1, 8, 128)[:, ::2], None),
    (t(1, 4, 128), t(1, 4, 128), t(1, 4)), (t(1, 4, 128), t(1, 4, 128), t(1, 4, dtype=F64)),
    (t(1, 4, 128), t(1, 4, 128), t(1, 4, dtype=torch.int32)), (t(1, 4, 128), t(1, 4, 128), t(4, 8, dtype=F32)[:, ::2])])
def test_tensors_of_attention(q, out, lse):
    with pytest.raises(ValueError):
        B.cart_q8_attention(0, 0, [0], q, out, lse)
    with pytest.raises(ValueError):
        B.cart_q8_decode_step(0, 0, [0], t(1, 2, 128), t(1, 2, 128), q, out, lse)


@pytest.mark.parametrize("k,v", [
    (t(3, 2, 128, dtype=HALF), t(3, 2, 128, dtype=HALF)), (t(3, 2, 128), t(3, 2, 128, dtype=F32)), (t(3, 2, 128), t(2, 2, 128)),
    (t(3, 2, 64), t(3, 2, 64)), (t(3, 256), t(3, 256)), (t(3, 2, 256)[..., ::2], t(3, 2, 256)[..., ::2]),
    (t(3, 2, 128), t(3, 4, 128)[:, ::2])])
def test_tensors_of_write(k, v):
    with pytest.raises(ValueError):
        B.cart_q8_write(0, 0, [0], [3], k, v)


def test_counts_and_reads():
    with pytest.raises(ValueError):
        B.cart_q8_write(0, 0, [0, 1], [3], t(3, 2, 128), t(3, 2, 128))
    with pytest.raises(ValueError):
        B.cart_q8_read(0, 0, [0], [0, 0], [3], t(3, 2, 128), t(3, 2, 128))
    with pytest.raises(ValueError):
        B.cart_q8_read(0, 0, [0], [0], [3], t(3, 2, 128), t(3, 2, 128, dtype=HALF))
    with pytest.raises(ValueError):
        B.cart_q8_decode_step(0, 0, [0], t(1, 2, 128, dtype=HALF), t(1, 2, 128), t(1, 4, 128), t(1, 4, 128))
