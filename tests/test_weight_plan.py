"""The launch plan of the accumulated weights, without a GPU: no launch is empty, and the batches that the GPU tests of
its variants use take the variants that they are there for."""
import random
import shutil

import pytest

from weight_plan import weight_plan

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ missing")


def _whole(p):
    """Every launch of the plan has workgroups, and a workspace where sums are joined, for all of them."""
    assert p.tiles > 0 and p.sink_tiles >= 0
    assert p.workspace > 0 if p.parts > 1 else p.workspace == 0
    assert p.sink_tiles > 0 or p.parts <= 1               # the join has a workgroup for each tile of sinks
    assert p.tiles + p.sink_tiles * p.parts <= 65535
    assert p.few or not p.ahead


@pytest.mark.parametrize("new", [1, 4, 5, 17, 272, 273, 700, 5000, 100000])
@pytest.mark.parametrize("window", [1, 16, 100, 1024])
@pytest.mark.parametrize("sink", [0, 1, 64, 65, 1024, 1025, 1 << 20])
def test_no_launch_is_empty(new, window, sink):
    p = weight_plan([new + 10, 10], [new, 1], 2, 4, window, sink)
    _whole(p)
    assert sink or p.parts <= 1


def test_no_launch_is_empty_over_random_batches():
    rng = random.Random(3)
    for _ in range(3000):
        log = lambda hi: int(hi ** rng.random())
        reqs = log(200)
        new = [log(20000) for _ in range(reqs)]
        lengths = [n + log(40000) - 1 for n in new]
        _whole(weight_plan(lengths, new, log(64), log(16), rng.choice([0, log(1 << 14), (1 << 31) - 1]),
                           rng.choice([-1, 0, 1, 4, log(4096), (1 << 31) - 1])))


def test_variants_of_few_rows():
    from test_gpu_sink_weights_variants import TILES
    t = dict(lengths=TILES["lengths"], new=TILES["new"], heads=TILES["heads"], group=2)
    for dim in (64, 128, 256):
        for window, sink in ((0, -1), (300, -1), (1200, 4), (300, 70), (1200, 0)):
            p = weight_plan(window=window, sink=sink, dim=dim, **t)
            assert p.few and p.ahead and p.tiles == 1, (dim, window, sink)
    assert not weight_plan(dim=80, **t).ahead and weight_plan(dim=80, **t).tiles == 6
    # a wave for each tile where requests may be ragged and there are few heads, or keys; else up to 2,048 keys a workgroup
    assert weight_plan([9000] * 2, [1] * 2, 8, 4)[1:5] == (True, False, 256, 36)
    assert weight_plan([511] * 1024, [1] * 1024, 8, 4)[1:5] == (True, False, 256, 2)
    assert weight_plan([4096] * 8, [1] * 8, 8, 4, dim=128)[1:5] == (True, False, 256, 16)
    assert weight_plan([32768] * 8, [1] * 8, 8, 4, dim=128)[1:5] == (True, True, 256, 32)
    assert weight_plan([16384] * 64, [1] * 64, 8, 4, dim=128)[1:5] == (True, True, 256, 8)
    assert weight_plan([32768], [1], 8, 4, dim=128)[1:5] == (True, True, 256, 64)
    assert weight_plan([32768], [1], 8, 4, dim=80)[1:5] == (True, False, 256, 128)
    assert weight_plan([8192] * 64, [1] * 64, 8, 4, window=2048, sink=4, dim=128)[1:5] == (True, True, 256, 1)


def test_tiles_of_many_rows():
    from test_gpu_sink_weights_variants import PAIRS
    for t, parts in zip(PAIRS, (1, 2)):
        for sink in (0, 4, 70):
            p = weight_plan(group=2, sink=sink, dim=64, **t)
            assert p.windowed and not p.few and p.keys == 128 and p.parts == (parts if sink else 1), (t, sink)
        assert weight_plan(group=2, sink=-1, **t).keys != 128
    rng = random.Random(4)
    for _ in range(2000):                                  # 128 keys: with the windowed kernels alone
        new = [rng.randint(1, 3000) for _ in range(rng.randint(1, 8))]
        p = weight_plan([n + rng.randint(0, 3000) for n in new], new, rng.randint(1, 128), 4, rng.choice([0, 500, 1024]), rng.choice([-1, 0, 4]))
        assert p.keys in (64, 256) or (p.keys == 128 and p.windowed)
