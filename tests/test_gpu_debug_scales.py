"""IKV_DEBUG=1 names an E4M3 scale that is not a power of two, in the decode and in the chunk
calls, where a token sees its row; int8 scales may be any number."""
import pytest

from paper_2606_09916_amd import ikv
from test_gpu_attend import Setup

pytestmark = pytest.mark.gpu

N, SINKS, WINDOW = 90, 2, 20


@pytest.mark.parametrize("n", [1, 3, 50])
@pytest.mark.parametrize("value", [3.0, 0.75, -0.5, 0.0, float("inf"), 2.0 ** -130, 1.0 / 448])
def test_scales_that_are_no_powers(dev, monkeypatch, n, value):
    import torch
    s = Setup(dev, "e4m3", "bf16", 2, 4, 2, 64, [N, N], n)
    q = s.queries(2 * n)
    run = lambda window=0: s.run(q, SINKS, window, decode=n == 1)  # noqa: E731
    want, narrow = run(), run(WINDOW)
    monkeypatch.setenv("IKV_DEBUG", "1")
    assert torch.equal(run(), want) and torch.equal(run(WINDOW), narrow)
    slots = s.live.long()
    old = s.sc.clone()
    # no token's window holds entry 2, the first after the sinks, of 90 with chunks of up to 50
    for entry, i, what in ((2, 0, "key"), (2, 1, "value")):
        s.sc[1, slots[N + entry], 1, i] = value
        with pytest.raises(ikv.IkvError, match=rf"session 1: the {what} scale of live\[{entry}\] .*layer 1, KV head 1") as e:
            run()
        assert e.value.status == -1
        assert torch.equal(run(WINDOW), narrow)
        s.sc.copy_(old)
    for entry in (0, N - 1):                             # a sink, and the newest entry
        s.sc[0, slots[entry], 0, 1] = value
        with pytest.raises(ikv.IkvError, match=rf"session 0: the value scale of live\[{entry}\]"):
            run(WINDOW)
        s.sc.copy_(old)
    s.sc[0, slots[N - 1], 0, 1] = float("nan")           # a row that was not finite when it was stored
    run()


def test_int8_scales_may_be_any(dev, monkeypatch):
    s = Setup(dev, "int8", "bf16", 1, 4, 2, 64, [N], 3)
    monkeypatch.setenv("IKV_DEBUG", "1")
    s.sc[:] = 3.0
    q = s.queries(3)
    s.check(s.run(q), q, [3])
