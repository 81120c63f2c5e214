"""A generation job whose prompt comes in chunks is the job whose prompt is there whole: the same keys and values to compress, the
same scores to rounding, and the same kept positions wherever the scores decide beyond it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def mods():
    from paper_2404_04793_amd import binding, session, workloads
    return binding, session, workloads


@pytest.mark.parametrize("policy", ["h2o", "streaming"])
@pytest.mark.parametrize("name,kw,ragged", [("tiny", dict(P=272), False), ("llama2_70b", dict(L=2, B=2, P=333, S=3, Hq=16, Hkv=2, hidden=256), False),
                                            ("llama2_7b", dict(L=2, B=3, P=200, S=3, Hq=4, Hkv=4, hidden=256), True)])
def test_session_with_the_prompt_in_chunks(mods, name, kw, ragged, policy):
    sqa, session, W = mods
    wl = W.scaled(W.WORKLOADS[name], policy=policy, **kw)
    lens = [wl.P - 37 * b for b in range(wl.B)] if ragged else None
    jobs = [session.Session(wl, DEV, prompt_len=lens, prompt_chunk=c) for c in (None, 64)]
    for s in jobs:
        s.run_pass()
        torch.cuda.synchronize()
    whole, parts = jobs
    if ragged:
        assert int(parts.status) == 0 == int(whole.status)
    for l in range(wl.L):
        for b in range(wl.B):
            n = lens[b] if ragged else wl.P
            assert torch.equal(whole.Kp[l][b, :, :n], parts.Kp[l][b, :, :n]) and torch.equal(whole.Vp[l][b, :, :n], parts.Vp[l][b, :, :n])
            if policy != "h2o":
                continue
            x, y = whole.scores[l][b, :, :n], parts.scores[l][b, :, :n]
            torch.testing.assert_close(x, y, rtol=1e-4, atol=1e-6)
    assert whole.budgets == parts.budgets
    if policy == "streaming":                     # no score decides anything: the same caches and outputs, bit for bit
        assert torch.equal(whole.out, parts.out)
        assert all(torch.equal(x, y) for x, y in zip(whole.caches.pos, parts.caches.pos))
    else:
        assert bool(torch.isfinite(parts.out.float()).all())
