"""grid_attend of more sequences times tiles of the longest chunk than a launch has workgroups: few of them have rows.
The same batch under a tighter bound of the chunks' lengths takes the same tiles: results have the same bits."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_gpu_attend import G, Batch, reference  # noqa: E402,F401

pytestmark = pytest.mark.gpu

LENS = [(i % 8, 8 + 13 * i % 90) for i in range(5000)]
LENS[7], LENS[2500], LENS[4999], LENS[0] = (700, 900), (300, 300), (77, 1000), (130, 200)


def bits(x):
    return [y.view(torch.int16 if y.element_size() == 2 else torch.int32) for y in x]


@pytest.mark.parametrize("window", [0, 50])
@pytest.mark.parametrize("heads", [(16, 1, 64), (16, 1, 128), (32, 2, 256)])
def test_tiles_by_rows(G, heads, window):  # noqa: F811
    bt = Batch(LENS, heads, 16, "bf16", seed=41)
    assert heads[1] * len(LENS) * (-(-bt.T * 16 // 128)) > 1 << 23
    out, lse = torch.full_like(bt.q, 7.0), torch.full((bt.T, bt.hq), 7.0, device="cuda")

    def same():
        want = bits(bt.attend(G, window=window, out=out.clone(), lse=lse.clone()))
        got = bits(bt.attend(G, window=window, out=out.clone(), lse=lse.clone(), max_q=1 << 24))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        return got

    got = same()
    # some sequences against the definition
    for b in (0, 1, 7, 2500, 4998, 4999):
        s = slice(int(bt.cu_host[b]), int(bt.cu_host[b + 1]))
        one = Batch([LENS[b]], heads, 16, "bf16", seed=41)
        one.k, one.v, one.q, one.table_host = bt.k, bt.v, bt.q[s], bt.table_host[b:b + 1]
        want, _, tol, _ = reference(one, window=window)
        assert bool(((got[0][s].view(torch.bfloat16).double() - want).abs() <= tol).all())
    # sequences that are bad: by their lengths, and from the first chunk that is not in order on
    bt.kv_len[9], bt.kv_len[2500] = 1 << 30, 3
    same()
    bt.cu[3001] = bt.cu[3000] - 1
    got = same()
    assert bool(torch.isnan(got[0][int(bt.cu_host[3000]):].view(torch.bfloat16).float()).all())
    # tokens before the first sequence and after the last
    bt.cu = torch.from_numpy(np.minimum(bt.cu_host + 500, bt.T).astype(np.int32)).cuda()
    same()
    bt.cu[0] = -1
    same()
