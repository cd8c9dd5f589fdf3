"""Attention whose streamed axis is split into so many parts, of so wide heads, that
their partial results are joined in rounds."""

import pytest

from .test_gpu_layer_ops import test_attention as attention
from .test_gpu_layer_ops import test_attention_gradient as gradient
from .test_gpu_layer_ops import test_same_bits_again_on_another_stream_and_replayed as same_bits

FWD = [
    dict(dtype="f32", n=1, m=500, d=208, heads=4),
    dict(dtype="f32", n=200, d=160, heads=2),
    dict(dtype="f16", n=1, m=500, d=256, heads=4),
    dict(dtype="bf16", n=1, m=5000, d=128, heads=4, batch=2, slopes=True, lengths=(5000, 2501)),
    dict(dtype="bf16", n=1, m=16305, d=128, heads=4, batch=2, slopes=True, lengths=(16305, 16300)),
    dict(dtype="f16", n=1, m=6000, d=96, heads=8, kv_heads=2, cap=8.0),
    dict(dtype="f32", n=2, m=1500, d=256, heads=2, causal=True),
]
GRAD = [
    dict(dtype="f32", n=300, d=72, heads=4, kv_heads=1),
    dict(dtype="f32", n=300, d=128, heads=4, kv_heads=1, causal=True),
    dict(dtype="f32", n=300, d=224, heads=4, kv_heads=1),
    dict(dtype="f16", n=300, d=256, heads=4, kv_heads=1),
    dict(dtype="bf16", n=300, d=208, heads=4, kv_heads=1, cap=6.0),
    dict(dtype="f32", n=33, m=2500, d=112, heads=2, causal=True, cap=10.0),
]
_id = lambda c: "-".join(f"{k}{v}" for k, v in c.items() if k != "lengths")  # noqa: E731


@pytest.mark.gpu
@pytest.mark.parametrize("case", FWD, ids=_id)
def test_attention_joined_in_rounds(case):
    attention(case)


@pytest.mark.gpu
@pytest.mark.parametrize("case", GRAD, ids=_id)
def test_gradients_joined_in_rounds(case):
    gradient(case)


@pytest.mark.gpu
@pytest.mark.parametrize("name,sizes", [
    ("mha", dict(heads=4, n=1, m=500, d=208, dtype="f32")),
    ("mha", dict(batch=2, heads=4, n=1, m=16305, d=128, dtype="bf16", slopes=True, lengths=True)),
    ("mha_grad", dict(heads=4, kv_heads=1, n=300, d=128, dtype="f16", causal=True, cap=8.0)),
    ("mha_grad", dict(heads=4, kv_heads=1, n=300, d=96, dtype="f32")),
], ids=str)
def test_joins_repeat_their_bits(name, sizes):
    same_bits(name, sizes)
