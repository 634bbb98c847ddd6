"""Attention behind shared prefixes rounds once, however many share one: its outputs are the 64-bit results' nearest values of their type, but for results that lie next to a border.

A value whose error before the rounding is e is rounded to the other side of a border with the probability |e| / ulp, and is an ulp off then: the mean square of the
difference from the rounded 64-bit result is |e| ulp, at most eps |e x|; over all values, with errors of the relative size d, its norm is at most sqrt(eps d) of the
result's. d is the sums' in fp32: (P + L) / 16 + 64 additions of 2^-24 each, 2^-17.0 for the sizes here, the scores' (sqrt(D + 4) roundings of random sign, 2^-23 of scores of about
1) and exponentials' (2^-22) are below that: sqrt(eps 2^-17) for fp16. bf16 has weights of 11 bits (2^-12.4 in the mean, 2^-12 at most), an eighth of its own rounding:
sqrt(eps 2^-12)."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import test_gpu_shared as shared
from test_gpu_shared import b  # noqa: F401


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,T", [(128, 64), (64, 16)])
@pytest.mark.parametrize("S,G,new", [(4, 4, 1), (16, 8, 1), (4, 8, 3), (3, 4, 20)])
@pytest.mark.parametrize("wide", [None, 4096])
def test_rounded_once(b, dtype, D, T, S, G, new, wide):  # noqa: F811
    """Groups of few and many rows, own tokens of few and many, in narrow tables and wide ones."""
    own = [new + 100 + 13 * s for s in range(S)]
    _, _, out, _, (ref, _) = shared.run(b, [600], [S], own, [new] * S, G, 2, D, T, dtype, seed=S + G, scale=1 / 64, widths=(None, wide and wide // T))
    off = float((out.double() - ref.to(dtype).double()).norm() / ref.norm())
    assert off <= math.sqrt(torch.finfo(dtype).eps * 2.0 ** (-17 if dtype == torch.float16 else -12)), f"{off:.3g}"
