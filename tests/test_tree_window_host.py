"""What grid_tree_masks_window refuses, and that it does nothing where there is nothing to do: through the C ABI with addresses
that are never read, and through the package's function on tensors in host memory."""

import pytest

from test_step_host import AT, S, refused  # noqa: F401
from test_tree_host import by, made


@pytest.mark.parametrize("name,bad", [("n_seqs", 0), ("n_seqs", 65536), ("n_tokens", -1), ("n_tokens", (1 << 24) + 1),
                                      ("max_q", 0), ("max_q", 1025), ("stride_words", 0), ("cu_q", None), ("parent", None),
                                      ("masks", None), ("depth", None)])
def test_bad_arguments(S, name, bad):  # noqa: F811
    refused(S, S.lib().grid_tree_masks_window(by(made("tree_masks", **{name: bad})), 5, None), "grid_tree_masks_window")


def test_windows(S):  # noqa: F811
    L = S.lib()
    for window in (-1, -2 ** 31):
        refused(S, L.grid_tree_masks_window(by(made("tree_masks")), window, None), "window")
    assert L.grid_tree_masks_window(None, 3, None) == -1
    for window in (0, 1, 2 ** 31 - 1):
        assert L.grid_tree_masks_window(by(made("tree_masks", n_tokens=0, parent=None, masks=None, depth=None)), window, None) == 0


def test_python_refusals(S):  # noqa: F811
    torch = pytest.importorskip("torch")
    parent, cu = torch.zeros(7, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for error, word, window in ((ValueError, "GPU", 3), (ValueError, "window", -1), (TypeError, "window", "x"),
                                (TypeError, "window", 2.5)):
        with pytest.raises(error, match=word):
            S.G.tree_masks(parent, cu, 7, window=window)
