"""Chunk attention with several row blocks and several splits at once, over sessions whose chunks
differ, on numbers of (session, layer, KV head) that are no multiple of the eight that the grid
deals out; and on many of them with none of it split."""
import pytest

from test_gpu_attend import Setup

pytestmark = pytest.mark.gpu

# L, Hq, Hkv, D, list lengths, tokens (a shorter list's chunk is the whole list)
CASES = [(1, 12, 3, 128, [90, 1500, 600], 150), (1, 8, 1, 64, [2000, 33], 300), (3, 2, 2, 64, [700, 1, 701], 333),
         (7, 16, 8, 64, [257, 64, 320], 64)]


@pytest.mark.parametrize("code,io", [("int8", "bf16"), ("e4m3", "bf16"), ("bf16", "bf16"), ("int8", "f32"), ("e4m3", "f32")])
@pytest.mark.parametrize("L,Hq,Hkv,D,lengths,n", CASES)
def test_blocks_and_splits(dev, code, io, L, Hq, Hkv, D, lengths, n):
    s = Setup(dev, code, io, L, Hq, Hkv, D, lengths, n, seed=L + n)
    q = s.queries(sum(s.ns))
    for sinks, window in ((0, 0), (70, 200)):
        s.check(s.run(q, sinks, window), q, s.ns, sinks, window)
