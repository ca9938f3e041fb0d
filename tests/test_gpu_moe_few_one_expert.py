"""The layer for a few tokens where one expert takes them all: four sets of 16 tokens on the same weights, in both types of
activations and of results, against the fp64 form and its bounds."""
import pytest
import torch

from gpu_util import require_gpu, say
from test_gpu_moe_few import DT, check, layer, routing, tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [16, 63, 64])
@pytest.mark.parametrize("d,f", [(2056, 520), (4096, 136), (264, 2056)])
@pytest.mark.parametrize("x,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
def test_all_tokens_on_one_expert(T, d, f, x, out):
    require_gpu()
    say(f"moe_few, one expert, T={T} d={d} f={f} {x} {out}")
    ids, w = routing(T, 2, 5)
    ids[:, 0], ids[:, 1] = 3, -1
    ids[T // 2] = torch.tensor([3, 3])  # twice
    ids[T // 3, 1] = 1                  # and another one
    check(tokens(T, d, x), ids, w, layer(5, d, f), DT[out])
