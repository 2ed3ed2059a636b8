"""Attention over the 4-bit cache where its work is shared: long sequences, many row tiles, many workgroups."""
import pytest
import torch

import paper_2504_13989_amd as rq
from test_gpu_kv4 import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,group,dtype", [(128, 1, "bf16"), (128, 8, "f16"), (128, 16, "bf16"), (64, 4, "bf16")])
def test_results_do_not_go_by_the_sums_asked_for(d, group, dtype):
    lens = [7001, 40, 3333, 2600]
    b = Batch(lens, 2, d, 64, True, seed=11)
    q, _ = b.queries([1] * 4, 2 * group, dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    plain = rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens)
    for _ in range(8):
        assert torch.equal(plain, rq.kv4_attention(b.h, b.cache, q, b.dev_table, b.dev_lens, lse=lse))
    b.check(q, [1] * 4, plain, lse)
