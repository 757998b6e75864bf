"""Workers of AD-PSGD that train a language policy with the operators of a training step (GPU only)."""
import numpy as np
import pytest

from paper_1710_06952_amd.studies import policy_model as S


def test_views_of_the_flat_vector():
    import torch
    p = S.Policy(11, 8, 5, 0, "cpu")
    x = torch.from_numpy(p.initial(0))
    assert x.numel() == p.d == 64 + 8 + 88 + 11
    parts = p.views(x)
    assert [tuple(v.shape) for v in parts] == p.shapes and torch.equal(torch.cat([v.reshape(-1) for v in parts]), x)
    assert parts[0].data_ptr() == x.data_ptr()


@pytest.mark.gpu
@pytest.mark.parametrize("loss,events,vocab", [("policy", 400, 64), ("preference", 200, 512)])
def test_the_right_answers_become_likely(loss, events, vocab):
    res = S.run_study(loss, n=4, vocab=vocab, width=64, prompts_each=16, M=64, events=events, gamma=5e-3, seed=1)
    print(res["chance"], res["losses"], flush=True)
    assert res["events"] == events == sum(res["steps"])
    assert np.isfinite(res["losses"]).all() and np.isfinite(res["chance"]).all()
    assert res["chance"][-1] > 5 * res["chance"][0]
    if loss == "preference":
        assert res["losses"][-1] < 0.5 * res["losses"][0]
    assert "quarter" in S.format_table(res)
