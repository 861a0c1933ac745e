"""Terms of the policy loss that do not count beside infinities: what a term multiplies by 0 is left out of the loss and its gradient, whatever the term itself is.
By every way in which the loss handles a row.  No tolerances: each call is compared with one that does not have the term, bit for bit."""
import gc

import pytest
import torch

from test_gpu_loss import BF16, FP32, Case, memory
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

# a few short rows by one workgroup; rows that a wavefront holds, a workgroup of 256, 512 and 1024 lanes; long rows by workgroups that stay; parts
SHAPES = [(9, 31, FP32), (40, 1000, BF16), (9, 10_003, BF16), (130, 20_003, BF16), (130, 40_001, FP32), (515, 32_773, FP32), (9, 70_001, BF16)]


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()
    yield
    torch.cuda.empty_cache()


def call(c, spec, **kw):
    stats, logprob = torch.full((4,), 7.0, device="cuda"), torch.full((c.rows,), 7.0, device="cuda")
    dx = torch.full_like(c.logits, 7.0)
    fo.policy_loss(spec, c.logits, c.tokens, c.advantages, stats, logprob=logprob, dlogits=dx, workspace=memory(fo.policy_loss_workspace(c.logits)), **kw)
    return stats, logprob, dx


@pytest.mark.parametrize("rows,vocab,dtype", SHAPES)
def test_a_kl_term_that_is_only_watched(rows, vocab, dtype):
    c = Case(rows, vocab, dtype, masked=0, seed=40)
    c.logits[1, c.tokens[1]] = float("-inf")                  # a token of probability 0, to which the reference gives a chance
    ref = (torch.randn(rows, generator=torch.Generator().manual_seed(vocab)) - 6).cuda()
    old = ref + 0.3
    ref[2] = 900.0                                            # so far above that the term overflows
    spec = fo.PolicyLoss(kl_weight=0.0)
    for kw in (dict(), dict(old_logprob=old), dict(weights=c.weights + 0.1)):
        without, with_ref = call(c, spec, **kw), call(c, spec, ref_logprob=ref, **kw)
        assert bool(torch.isfinite(without[0]).all()) and bool(torch.isfinite(without[2]).all()) and float(without[0][2]) == 0
        for k in (0, 1, 3):
            assert torch.equal(with_ref[0][k], without[0][k]), k
        assert float(with_ref[0][2]) == float("inf")
        assert torch.equal(with_ref[1], without[1]) and torch.equal(with_ref[2], without[2])
    # a term with a weight is infinite all the same
    assert float(call(c, fo.PolicyLoss(kl_weight=0.1), ref_logprob=ref)[0][0]) == float("inf")


@pytest.mark.parametrize("rows,vocab,dtype", SHAPES)
def test_an_advantage_of_0_has_no_surrogate(rows, vocab, dtype):
    c = Case(rows, vocab, dtype, masked=0, seed=41)
    c.advantages[1:4] = 0
    old = (torch.randn(rows, generator=torch.Generator().manual_seed(vocab)) - 6).cuda()
    ref = old + 0.2
    old[1], old[2] = float("-inf"), -2000.0                   # ratios that are infinite, by their definition or in FP64
    w = c.weights + 0.1
    without = w.clone()
    without[1:3] = 0
    got, want = (call(c, fo.PolicyLoss(), old_logprob=old, weights=v) for v in (w, without))
    assert bool(torch.isfinite(got[0]).all()) and torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    assert bool(torch.isfinite(got[1]).all()) and torch.equal(got[1][3:], want[1][3:])
    # the KL term is there all the same
    spec = fo.PolicyLoss(kl_weight=0.1)
    got, want = call(c, spec, old_logprob=old, ref_logprob=ref, weights=w), call(c, spec, old_logprob=ref, ref_logprob=ref, weights=w)
    assert torch.equal(got[2][1:3], want[2][1:3]) and bool((got[2][1:3] != 0).any(1).all()) and bool(torch.isfinite(got[0]).all())
    # and what is no number stays none
    old[3] = float("nan")
    got = call(c, fo.PolicyLoss(), old_logprob=old, weights=w)
    assert bool(torch.isnan(got[0][0])) and bool(torch.isnan(got[2][3]).all())


def test_rows_of_negative_tokens_have_no_weight_in_a_preference_loss():
    # it sees no tokens: their logprob of 0 less the reference's is left out by the weight alone
    c = Case(40, 300, BF16, masked=0.4, seed=42)
    ref = (torch.randn(40, generator=torch.Generator().manual_seed(1)) - 6).cuda()
    wide = torch.empty(40, dtype=torch.float64, device="cuda")
    fo.token_logprob(c.logits, c.tokens, logprob64=wide, workspace=memory(fo.token_logprob_workspace(c.logits)))
    there = c.tokens >= 0
    cuts = torch.tensor([0, 9, 20, 33, 40], device="cuda")
    kept = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), there.long().cumsum(0)])[cuts]
    spec, loss, margins = fo.PreferenceLoss(), torch.empty(3, device="cuda"), torch.empty(3, 2, device="cuda")
    slopes, some = torch.empty(40, device="cuda"), torch.empty(int(there.sum()), device="cuda")
    fo.preference_loss(spec, wide, cuts, loss[:1], ref_logprob=ref, weights=there.float(), margins=margins[0], dlogprob=slopes)
    fo.preference_loss(spec, wide[there], kept, loss[1:2], ref_logprob=ref[there], margins=margins[1], dlogprob=some)
    # (the same values in FP64 sums of another order)
    assert torch.allclose(margins[0], margins[1], rtol=2.0 ** -22, atol=0) and torch.allclose(loss[0], loss[1], rtol=2.0 ** -22, atol=0)
    assert torch.allclose(slopes[there], some, rtol=2.0 ** -22, atol=0) and not bool(slopes[~there].any())
    fo.preference_loss(spec, wide, cuts, loss[2:], ref_logprob=ref, margins=margins[2])
    assert bool(((margins[2] - margins[0]).abs() > 0.1).all())
