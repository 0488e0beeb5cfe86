"""Appends of many tokens, several to a workgroup: loads that run ahead, places and angles of every token of the group,
padding in the middle of one and a short last one."""
import pytest
import torch

from serving_common import Case
from test_gpu_serving import check_append

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("new,lens,first,extra,dtype,norm", [
    ([3, 700, 1, 250, 0, 1090], [3, 900, -1, 260, 5, 1090], 3, 4, "bf16", True),            # 2051 tokens, two a workgroup
    ([1900, 2, 1187], [1700, 2, 5000], 0, 11, "f16", False),                                # 3100 tokens, three
    ([1, 1, 1, 2500, 7, 1593], [9, -1, 0, 2501, -3, 1600], 1, 0, "f16", True),              # 4104 tokens, four
])
def test_several_tokens_a_workgroup(new, lens, first, extra, dtype, norm):
    from paper_2609_17184_amd import serving
    c = Case(252, 2, 64, 48, dtype, new, lens, 1000, seed=len(new), first=first, extra=extra)
    g = torch.Generator().manual_seed(5)
    qn, kn = ((1 + 0.3 * torch.randn(64, generator=g)) if norm else None for _ in range(2))
    out = torch.full(c.q.shape, 3.0, dtype=c.dtype, device=DEV)
    before = out.cpu()
    serving.rope_append(c.q.to(DEV), c.kn.to(DEV), c.vn.to(DEV), c.cache, c.batch, serving.rope_frequencies(32),
                        q_norm=None if qn is None else qn.to(DEV), k_norm=None if kn is None else kn.to(DEV), eps=1e-5,
                        out=out)
    check_append(c, 32, (qn, kn), 1e-5, out, before)
