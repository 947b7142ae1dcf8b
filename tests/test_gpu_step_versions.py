"""Tensors that the calls of a model's step write are known to torch as written: a backward pass that needs what they held
refuses instead of using what they hold now."""

import pytest

torch = pytest.importorskip("torch")

from test_gpu_attend import G, Batch  # noqa: E402,F401
from test_gpu_verify import Case, pack  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def bumped(tensors, call):
    before = [t._version for t in tensors]
    call()
    return [t._version > v for t, v in zip(tensors, before)]


def test_versions(G):  # noqa: F811
    bt = Batch([(2, 40), (1, 900)], (4, 2, 64), 16, "bf16", seed=1)
    k = bt.rand((bt.T, 2, 64))
    status, q_out = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros_like(bt.q)
    written, read = [bt.k, bt.v, status, q_out], [k, bt.q, bt.table, bt.kv_len, bt.cu]
    call = lambda: G.kv_append(k, k, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, q=bt.q, q_out=q_out, status=status)  # noqa: E731
    assert bumped(written + read, call) == [True] * 4 + [False] * 5
    out, lse = torch.zeros_like(bt.q), torch.zeros((bt.T, 4), device="cuda")
    work = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    call = lambda: bt.attend(G, out=out, lse=lse, workspace=work)  # noqa: E731
    assert bumped([out, lse, work, bt.k, bt.v, bt.q], call) == [True] * 3 + [False] * 3
    c = Case(2, 1, 50, seed=2)
    made = [x.cuda() for x in (torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2))]
    call = lambda: c.run(G, tokens=made[0], accepted=made[1], logprobs=made[2], workspace=work)  # noqa: E731
    assert bumped(made + [work, c.logits], call) == [True] * 4 + [False]


def test_a_saved_tensor_is_missed(G):  # noqa: F811
    bt = Batch([(2, 40)], (4, 2, 64), 16, "bf16", seed=3)
    k = bt.rand((bt.T, 2, 64))
    x = torch.ones((), device="cuda", dtype=torch.bfloat16, requires_grad=True)
    loss = (x * bt.k).sum()  # keeps the pages for x's gradient
    G.kv_append(k, k, bt.k, bt.v, bt.table, bt.kv_len, bt.cu)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_in_inference_mode(G):  # noqa: F811
    with torch.inference_mode():
        bt = Batch([(2, 40)], (4, 2, 64), 16, "bf16", seed=4)
        k = bt.rand((bt.T, 2, 64))
        G.kv_append(k, k, bt.k, bt.v, bt.table, bt.kv_len, bt.cu, q=bt.q, q_out=bt.q)
        assert bt.attend(G)[0].shape == bt.q.shape
