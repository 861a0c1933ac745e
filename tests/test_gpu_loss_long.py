"""The policy loss of many rows so long that a compute unit holds one at a time, against its definition in 64 bits: rows of other lengths, at any address, rows
that do not count between ones that do, in place, and the same from a graph.  Tolerances as in test_gpu_loss.py."""
import gc

import pytest
import torch

from test_gpu_loss import BF16, FP32, Case, memory, policy
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,vocab,dtype,pad,shift", [
    (512, 65_544, BF16, 0, 0),           # one word more than the shape below holds
    (513, 65_551, BF16, 3, 5),           # odd rows at odd addresses
    (1030, 32_773, FP32, 1, 3),          # the last workgroups have a row more
    (512, 65_536, FP32, 0, 0),           # a full row
])
def test_long_rows(rows, vocab, dtype, pad, shift):
    policy(Case(rows, vocab, dtype, temperature=1.3, pad=pad, shift=shift, masked=0.4, seed=30))


@pytest.mark.parametrize("old,kl", [(False, None), (True, None)])
def test_long_rows_in_place(old, kl):
    policy(Case(520, 32_779, FP32, masked=0.1, seed=31), old=old, kl=kl, weights=False, in_place=True)


def test_long_rows_without_a_gradient_or_without_any_that_counts():
    policy(Case(512, 32_773, FP32, masked=0.2, seed=32), grad=False)
    c = Case(512, 32_773, FP32, masked=1.1, seed=33)
    c.logits.fill_(float("nan"))
    stats, logprob, dx = (torch.full(s, 7.0, device="cuda") for s in ((4,), (512,), (512, 32_773)))
    fo.policy_loss(fo.PolicyLoss(), c.logits, c.tokens, c.advantages, stats, logprob=logprob, dlogits=dx,
                   workspace=memory(fo.policy_loss_workspace(c.logits)))
    assert not (stats.any() or logprob.any() or dx.any())


def test_long_rows_without_a_result():
    c = Case(512, 32_773, FP32, masked=0.0, seed=34)
    # NaN, +infinity, nothing but -infinity, a token that is not there, and a mask beside them
    c.logits[1, 7], c.logits[2, 32_772], c.logits[3] = float("nan"), float("inf"), float("-inf")
    c.tokens[4] = 32_773
    c.logits[5, 1:] = float("-inf")
    c.tokens[5] = 0
    stats, logprob, dx = (torch.full(s, 7.0, device="cuda") for s in ((4,), (512,), (512, 32_773)))
    fo.policy_loss(fo.PolicyLoss(), c.logits, c.tokens, c.advantages, stats, logprob=logprob, dlogits=dx,
                   workspace=memory(fo.policy_loss_workspace(c.logits)))
    assert bool(torch.isnan(stats[0]))
    bad = torch.isnan(logprob)
    assert bad[1:5].all() and int(bad.sum()) == 4 and float(logprob[5]) == 0.0
    assert bool(torch.isnan(dx[1:5]).all()) and not bool(torch.isnan(dx[5:]).any()) and not bool(torch.isnan(dx[0]).any())
    assert float(dx[5].abs().max()) == 0.0


def test_long_rows_from_a_graph():
    c = Case(600, 40_003, FP32, masked=0.3, seed=35)
    first = [t.clone() for t in policy(c)]
    out = [torch.empty_like(t) for t in first]
    ws = memory(fo.policy_loss_workspace(c.logits))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fo.policy_loss(c.spec, c.logits, c.tokens, c.advantages, out[0], old_logprob=c.old, ref_logprob=c.ref, weights=c.weights, logprob=out[1],
                       dlogits=out[2], workspace=ws)
    for _ in range(3):
        for t in out:
            t.fill_(7.0)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, out))
