"""The calls of a model's step have no derivatives: tensors that want one are refused while torch records them.  On
tensors in host memory, which are refused for that in the end."""

import pytest

torch = pytest.importorskip("torch")

from test_step_host import S  # noqa: E402,F401

half = torch.bfloat16


def calls(G):
    """(call, its arguments, the names of those that a derivative could be asked of)"""
    pages, table = torch.zeros(4, 16, 2, 64, dtype=half), torch.zeros(3, 5, dtype=torch.int32)
    lens, cu = torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    k, q = torch.zeros(7, 2, 64, dtype=half), torch.zeros(7, 6, 64, dtype=half)
    yield G.kv_append, dict(k=k, v=k.clone(), k_pages=pages, v_pages=pages.clone(), block_table=table, kv_len=lens, cu_q=cu,
                            q=q, q_out=q.clone(), cos=torch.zeros(9, 32), sin=torch.zeros(9, 32), q_norm=torch.zeros(64),
                            k_norm=torch.zeros(64)), ["k", "v", "k_pages", "v_pages", "q", "q_out", "cos", "sin", "q_norm",
                                                      "k_norm"]
    yield G.attend, dict(q=q, k_pages=pages, v_pages=pages.clone(), block_table=table, kv_len=lens, cu_q=cu, max_q=7,
                         max_kv=80, out=q.clone(), lse=torch.zeros(7, 6)), ["q", "k_pages", "v_pages", "out", "lse"]
    yield G.verify, dict(logits=torch.zeros(2, 4, 40), draft=torch.zeros(2, 3, dtype=torch.int32),
                         draft_probs=torch.zeros(2, 3, 40), uniform=torch.zeros(2, 3), noise=torch.zeros(2, 40),
                         temperature=torch.zeros(2), logprobs=torch.zeros(2, 4)), ["logits", "draft_probs", "uniform",
                                                                                   "noise", "temperature", "logprobs"]


def test_tensors_that_require_a_gradient(S):  # noqa: F811
    for call, args, names in calls(S.G):
        for name in names:
            kw = {**args, name: args[name].clone().requires_grad_()}
            with pytest.raises(RuntimeError, match="gradient"):
                call(**kw)
            with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
                call(**kw)
            with torch.inference_mode(), pytest.raises(ValueError, match="GPU"):
                call(**kw)
            kw[name] = kw[name].detach()
            with pytest.raises(ValueError, match="GPU"):
                call(**kw)


def test_tensors_with_a_tangent(S):  # noqa: F811
    import torch.autograd.forward_ad as fwd
    for call, args, names in calls(S.G):
        for name in names:
            with fwd.dual_level():
                kw = {**args, name: fwd.make_dual(args[name], torch.ones_like(args[name]))}
                with pytest.raises(RuntimeError, match="gradient"):
                    call(**kw)
