"""An infinite value reaches a token as the infinity whatever the weight it has, down to 2^-126."""
import pytest
import torch

from paper_2402_17764_b200 import binding as B
from test_gpu_attention_shared import shared

pytestmark = pytest.mark.gpu

LN_2 = 0.6931471805599453  # as a scale: in fp32 it makes the factor between q . k and the power of two 1, so weights are 2^(q . k)


@pytest.mark.parametrize("power", [-1, -24, -60, -102, -109, -110, -117, -118, -125, -126])
@pytest.mark.parametrize("own", [[100, 80], [128, 128]])
def test_weights_that_are_powers_of_two(power, own):
    s, of = shared([(64, own)], 1, 64, 16, 16, 1)
    keys, values = s.pools[0].view(-1, 64), s.pools[1].view(-1, 64)
    for b, n in enumerate(own):
        i = torch.arange(n, device="cuda")
        row = s.table[b].long()[i // 16] * 16 + i % 16
        keys[row], values[row] = 0.0, 0.0
        keys[row, 0] = -200.0  # no weight
        keys[row[0], 0], values[row[0]] = 0.0, 1.0
        keys[row[37], 0], values[row[37], 3], values[row[37], 9] = float(power), float("inf"), float("-inf")
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    got = [B.attend_decode(cache, batch, q, scale=LN_2), B.attend_decode_shared(cache, batch, of, q, scale=LN_2, share_from=0)]
    cache.check()
    rest = torch.ones(64, dtype=torch.bool, device="cuda")
    rest[[3, 9]] = False
    want = 1.0 / (1.0 + 2.0 ** power)
    for out in got:
        assert torch.all(out[..., 3] == float("inf")) and torch.all(out[..., 9] == float("-inf"))
        # (the weights' sum in fp32, a quotient, and the rounding to bf16)
        assert torch.all((out[..., rest].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -15) * want)
