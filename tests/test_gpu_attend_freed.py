"""grid_attend under a window whose earlier pages are no longer in the block table: results keep their bits."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attend import G, Batch, agree  # noqa: E402,F401

pytestmark = pytest.mark.gpu

# lengths, and which launch they reach: all keys at once; shares and their joining (32 and 64 rows); tiles of 128 rows; the
# same split and joined
LAUNCHES = {"direct": ([(1, 400), (5, 130), (2, 333)], 40), "shares": ([(1, 1400), (5, 2130), (2, 333)], 900),
            "shares of 64": ([(12, 1400), (5, 2130), (2, 333)], 900), "tiles": ([(200, 2700), (5, 130)] * 30, 1100),
            "split": ([(90, 5000), (5, 3130)], 1500)}


@pytest.mark.parametrize("gone", [-1, 1 << 30])
@pytest.mark.parametrize("page", [4, 16, 48, 100])
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 1, 64), (4, 1, 256)])
@pytest.mark.parametrize("launch", LAUNCHES)
def test_pages_behind_the_window(G, launch, heads, page, gone):
    lens, window = LAUNCHES[launch]
    bt = Batch(lens, heads, page, "bf16", seed=page)
    want = bt.attend(G, window=window)
    agree(want, bt, window=window)
    some = 0
    for b, (n, kv) in enumerate(lens):
        behind = max(0, kv - n - window + 1) // page  # pages that end before the first position seen
        bt.table[b, :behind] = gone
        some += behind
    assert some
    got = bt.attend(G, window=window)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("launch", LAUNCHES)
def test_the_first_page_of_the_window_is_needed(G, launch):
    lens, window = LAUNCHES[launch]
    bt = Batch(lens, (8, 2, 128), 16, "bf16", seed=2)
    for b, (n, kv) in enumerate(lens):
        bt.table[b, max(0, kv - n - window + 1) // 16] = -1
    out, lse = bt.attend(G, window=window)
    first = torch.from_numpy(bt.cu_host[:-1][np.diff(bt.cu_host) > 0].astype(np.int64)).cuda()
    assert bool(torch.isnan(out[first].float()).all()) and bool(torch.isnan(lse[first]).all())
