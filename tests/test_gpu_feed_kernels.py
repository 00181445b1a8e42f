"""The kernels that the rules pick for serving sizes: the logits' slices and their sums of biases, tiles of many channels, the persistent gated block's
shares of the XCDs, sums at the ends of their bits.  Bit for bit against the definitions in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

import feed_util as U
from test_gpu_decoder import libs, same
from test_gpu_feed import DeviceLogits, ran, run


# ------------------------------------------------------------------------------------------- logits
def check_logits(c, kernel, what, off=0, in_place=False):
    torch, G, B = libs()
    G.say("logits: %s, at %d%s" % (what, off, ", in place" if in_place else ""))
    d = DeviceLogits(c, off, in_place)
    d.call()
    torch.cuda.synchronize()
    ran("logits_adjust_kernel<%d>" % kernel)
    if in_place:
        same(d.x, U.logits_by_rows(c, c.x), what)
    else:
        same(d.y[:c.y0.size], U.logits_by_rows(c), what)
        assert bool((d.y[c.y0.size:] == 77).all()), "wrote past the end: " + what


def wide_values(seed, n):
    """Biases of which a few take a row's sums beyond 32 bits."""
    rng = np.random.default_rng(seed)
    v = rng.integers(-500, 500, n).astype(np.int32)
    v[rng.random(n) < 0.02] = U.LOW
    v[rng.random(n) < 0.02] = U.HIGH
    return v


# rows x vocabulary whose slices have 2048 or 4096 tokens; ends of a slice, of half a slice and of neither; 16-byte rows and others
SLICED = [(3, 1030, 2048), (2, 2048, 2048), (5, 5121, 2048), (2, 7000, 2048), (64, 33000, 4096), (130, 16388, 4096), (136, 17001, 4096), (128, 14336, 4096)]


@pytest.mark.parametrize("rows,vocab,kernel", SLICED)
def test_logits_sums_of_biases_beyond_32_bits(gpu, rows, vocab, kernel):
    rng = np.random.default_rng(vocab)
    for off, in_place in ((0, False), (1, False), (0, True)):
        blens = rng.integers(0, 700, rows)
        blens[0], blens[-1] = 1500, 3
        c = U.Logits(vocab, rng.integers(0, 300, rows), vocab, blens, 3)
        c.values[:] = wide_values(vocab, c.values.size)
        c.ids[:40] = rng.integers(0, vocab)               # forty of one token, whose sum passes 32 bits on the way
        c.values[:40:2], c.values[1:40:2] = U.LOW, U.HIGH
        check_logits(c, kernel, "%d x %d, wide biases" % (rows, vocab), off, in_place)


def test_logits_a_long_list_of_biases_is_gone_through_a_fixed_number_of_times(gpu):
    # one value beyond 2^31 / n among n = 60000: once more for each half of a slice, where a walk for every token it holds would take the list's length squared
    torch, G, B = libs()
    rows, vocab, n = 4, 30000, 60000
    c = U.Logits(1, [100] * rows, vocab, [n] * rows, 2)
    c.values[:] = np.random.default_rng(2).integers(-500, 500, c.values.size)
    times = []
    for ban in (False, True):
        if ban:
            c.values[c.bstart[:-1] + 5] = U.LOW
            c.ids[c.bstart[:-1] + 5] = 77
        check_logits(c, 2048, "60000 biases a row%s" % (", one token banned" if ban else ""))
        d = DeviceLogits(c)
        best = 1e9
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(4):
                d.call()
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        times.append(best)
    assert times[1] < 8 * times[0], times             # (three walks for one, and beside them the same work)
