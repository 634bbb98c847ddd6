"""Own contexts of more tokens than a warp of the kernel of short contexts looks up at a time (512), around that border and the lengths where another kernel takes over (512 tokens of a
table for up to 32 sequences, 1024 for more). Bounds: tests/test_gpu_shared.py."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import test_gpu_shared as shared
from test_gpu_shared import b  # noqa: F401

F16, BF16 = torch.float16, torch.bfloat16
LENGTHS = [511, 512, 513, 527, 1000, 1023, 1024, 544, 1, 31, 33, 528, 480, 992, 1008, 64]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,T", [(128, 16), (64, 256), (64, 16), (128, 256)])
@pytest.mark.parametrize("groups", [[40], [8, 8, 0, 7, 8, 8]])
def test_two_windows(b, dtype, D, T, groups):  # noqa: F811
    """40 sequences of one token each: one group of many rows, and groups of few; the last of six has a sequence in front and none behind."""
    first = 40 - sum(groups)
    shared.run(b, [130 + 64 * i for i in range(len(groups))], groups, [LENGTHS[s % 16] for s in range(40)], [1] * 40, 4, 2, D, T, dtype, seed=T, first=first, widths=(None, 1024 // T))


@pytest.mark.parametrize("D,T", [(128, 64), (64, 16)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("groups", [[36], [9, 9, 9, 9]])
def test_several_new_tokens_across_the_border(b, D, T, causal, groups):  # noqa: F811
    new = [1 + s % 7 for s in range(36)]
    own = [max(n, x) for n, x in zip(new, [512 + s % 6 for s in range(20)] + [LENGTHS[s] for s in range(16)])]
    shared.run(b, [200] * len(groups), groups, own, new, 2, 2, D, T, F16, seed=D, causal=causal, widths=(None, 1024 // T))


@pytest.mark.parametrize("S", [32, 33])
@pytest.mark.parametrize("wide", [512, 528, 1024, 1040])
@pytest.mark.parametrize("G", [1, 8])
def test_either_side_of_the_limits(b, S, wide, G):  # noqa: F811
    own = [wide - s if s < 4 else 1 + 37 * s % wide for s in range(S)]
    shared.run(b, [300], [S], own, [1] * S, G, 2, 128, 16, BF16, seed=S, widths=(None, wide // 16))
