"""Groups that are whole powers of two of the sixteen lanes' experts stay in registers: every width of them (1, 2, 4
and 8 lanes a group), beside widths that go through LDS, with ties and with groups that are masked whole."""

import pytest
import torch

from .gpu_common import DEV
from .test_gpu_route_experts import check, make

pytestmark = pytest.mark.gpu

# N = 16 R experts, R = 2, 4, 8 or 16 a lane; 2, 4, 8 or 16 groups: 8, 4, 2 or 1 lanes each
GROUPS = [(N, G, keep) for N in (32, 64, 128, 256) for G in (2, 4, 8, 16) for keep in sorted({1, G // 2 + (G == 8), G - 1})]


@pytest.mark.parametrize("N,G,keep", GROUPS + [(48, 2, 1), (120, 4, 3), (240, 5, 2)])
@pytest.mark.parametrize("kind", ["plain", "ties", "masked groups"])
def test_groups_of_every_width(N, G, keep, kind):
    K = min(6, keep * (N // G))
    for dtype in (torch.float32, torch.bfloat16):
        logits = make(67, N, dtype, N + G, "ties" if kind != "plain" else kind)
        if kind == "masked groups":
            logits.view(67, G, N // G)[::2, 0] = -float("inf")
            logits.view(67, G, N // G)[::3, G - 1] = float("nan")
            logits.view(67, G, N // G)[1::4, :, 1:] = -float("inf")           # one live expert a group
            logits[5::11] = -float("inf")
        bias = torch.round(8 * torch.randn(N, generator=torch.Generator().manual_seed(G))) / 32
        for top2 in (False, True):
            for b in (None, bias.to(DEV)):
                check(logits.to(DEV), K, score="sigmoid" if top2 else "softmax", select_bias=b, groups=G, keep_groups=keep,
                      group_top2=top2, renorm=not top2)
