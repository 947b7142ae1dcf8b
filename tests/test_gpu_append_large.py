"""grid_kv_append of as many tokens as a call may have: entries are copied, so the cache holds the inputs' bits."""

import pytest

torch = pytest.importorskip("torch")

from test_gpu_attend import G  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,with_status", [(1 << 24, False), (1 << 24, True), ((1 << 24) - 1, True),
                                                ((1 << 23) + 1, False), (1 << 23, True)])
def test_the_most_tokens(G, tokens, with_status):  # noqa: F811
    page, before = 65536, 5
    k, v = (torch.randint(-(1 << 15), 1 << 15, (tokens, 1, 8), dtype=torch.int16, device="cuda").view(torch.bfloat16)
            for _ in range(2))
    pages = -(-(tokens + before) // page)
    k_pages, v_pages = (torch.zeros((pages, page, 1, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None]
    kv_len = torch.tensor([tokens + before], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda") if with_status else None
    G.kv_append(k, v, k_pages, v_pages, table, kv_len, cu, status=status)
    for x, into in ((k, k_pages), (v, v_pages)):
        got = into.flip(0).reshape(-1, 1, 8).view(torch.int16)
        assert torch.equal(got[before:before + tokens], x.view(torch.int16))
        assert not got[:before].any() and not got[before + tokens:].any()
    assert status is None or status.tolist() == [0]
