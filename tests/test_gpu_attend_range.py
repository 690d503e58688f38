"""Attention over values near the end of their type."""
import pytest
import torch

import cache_cases as cc

pytestmark = pytest.mark.gpu


def run(c, **kw):
    from paper_2408_05235_amd import api
    return api.tl_attend(c["q"], c["k"], c["v"], c["table"], c["length"], c["offset"], window=c["window"],
                         sinks=c["sinks"], want_lse=True, **kw)


@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("split", [False, True])
def test_values_near_the_end_of_bf16(gpu, new, dim, split):
    """A token of twice 2^124 with nearly all the weight, found after others:
    the sums hold it as long as sum w |v| does for weights of at most 1."""
    L = 3000 if split else 200
    c = cc.make(22, "bf16", 2, 1, dim, 16, [L], [new])
    kb, vb = c["dense"][0]
    kb.zero_()
    vb.fill_(1.0)
    at = 150
    kb[at, 0, 3] = 5.4375                       # 2^7.85 of the others' weight
    vb[at, 0] = 2.0 ** 125
    t = torch.arange(L + new)
    page = c["table"][0].cpu().long()[t // 16].cuda()
    c["k"][page, :, (t % 16).cuda()], c["v"][page, :, (t % 16).cuda()] = kb.cuda(), vb.cuda()
    c["q"] = torch.zeros(new, 2, dim, dtype=torch.bfloat16, device="cuda")
    c["q"][:, :, 3] = 1.0
    kw = {} if split else dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    out, lse = run(c, scale=1.0, **kw)
    cc.check(c, out, lse, scale=1.0)
