"""What the cache's status word reports, and when."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["append", "decode", "prompt"])
def test_check_waits_for_calls_on_every_stream(call):
    """The call that meets a bad page runs on a side stream, behind work that takes about 50 ms; check() is asked on the
    default stream at once, and leaves a status word that is clear for the next call."""
    s = R.Setup([40, 40], 2, 64, 16, 16, seed=71)
    s.table[1, 2] = s.n_pages
    cache = s.cache()
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    batch = B.KVBatch(s.table, s.kv_lens, cu if call == "prompt" else None)
    q, kv = rows(2, 4, 64, 72), rows(2, 2, 64, 73)
    out, ws = torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda"), B.alloc_attend_workspace(4, 2, 64, prompt=call == "prompt")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        if call == "append":
            B.kv_append(cache, batch, kv, kv, stream=side)
        else:
            (B.attend_prompt if call == "prompt" else B.attend_decode)(cache, batch, q, out=out, workspace=ws, stream=side)
        with pytest.raises(B.BitLinearError) as e:
            cache.check()
        assert e.value.status == B.ERR_PAGE
        torch.cuda.synchronize()
        assert cache.status.item() == B.OK
