"""How near the losses on logits come to their definitions in 64 bits, by bounds that follow the kernels' own sums, with u = 2^-24.

A power of two stands for exp((x - m) / T): the difference is off by u of itself, the product with the factor's two parts by u, so that the power is off by
2 u |x - m| / T, and by 2 u of its own.  A lane adds up eight values in three roundings (four in two) and at most 16 words of these in as many, in FP32; all else
is FP64, but a part's sum is brought to another largest value at most HOPS times, each by a power of 2 u, whose exponents add up to |x - m|.  So a value's part
of the sum is off by (2 |x - m| / T + ADDS) u of itself with ADDS = 2 (1 + HOPS) + 19.  HOPS: the words of a row of 262147 BF16 values lie 4096 or fewer to a pass of a
workgroup, which makes eight passes, once between its wavefronts, and once more between parts.

The largest value's own part is exact (its power is 1, words that hold a value of some weight are added up in FP64): beside a token that is all but certain only the others' part is off,
by as much of itself, and FP64 sums of fewer than 1000 additions by 2^-43."""
import gc

import pytest
import torch

import loss_reference as R
from test_gpu_loss import BF16, FP32, Case, check_logprob, forward, memory, policy
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

U = R.U
HOPS = 10
ADDS = 2 * (1 + HOPS) + 19


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()
    yield
    torch.cuda.empty_cache()


@pytest.fixture
def tight(monkeypatch):
    """The bounds of loss_reference.py, 3 sum p |x - m| / T + 2 + 1.5 adds, with the additions that there are."""
    monkeypatch.setattr(R, "adds", lambda vocab: (ADDS - 2) / 1.5)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,vocab", [(5, 1000), (5, 8192), (5, 50_257), (5, 131_073), (5, 262_147), (300, 4099), (300, 30_001), (260, 70_001)])
def test_log_probabilities(rows, vocab, dtype, tight):
    check_logprob(Case(rows, vocab, dtype, temperature=0.7, masked=0.1, seed=50))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,vocab", [(6, 9), (6, 1000), (6, 8192), (6, 50_257), (6, 262_147), (300, 4099), (300, 30_001), (260, 70_001)])
def test_tokens_that_are_all_but_certain(rows, vocab, dtype):
    c = Case(rows, vocab, dtype, masked=0, seed=51, spread=1.0)
    g = torch.Generator().manual_seed(vocab)
    row = torch.arange(rows)
    # ahead of the others by 16 to 36: probabilities of 1 - 10^-2 (of many others) to 1 - 10^-14
    ahead = 16 + 20 * torch.rand(rows, generator=g)
    tokens = c.tokens.cpu()
    x = c.logits.cpu()
    x[row, tokens] = (x.float().amax(1) + ahead).to(dtype)
    c.logits.copy_(x)
    x = x.double()
    gap = x[row, tokens][:, None] - x
    other = torch.exp(-gap)
    other[row, tokens] = 0
    want = -torch.log1p(other.sum(1))
    err = U * (other * (2 * gap + ADDS)).sum(1) + 2.0 ** -43
    wide = torch.full((rows,), 7.0, dtype=torch.float64, device="cuda")
    fo.token_logprob(c.logits, c.tokens, logprob64=wide, workspace=memory(fo.token_logprob_workspace(c.logits)))
    R.close(wide, want, err, "logprob64")
    # the policy loss's own sum, by its shape
    stats, logprob = torch.empty(4, device="cuda"), torch.empty(rows, device="cuda")
    fo.policy_loss(fo.PolicyLoss(), c.logits, c.tokens, c.advantages, stats, logprob=logprob, workspace=memory(fo.policy_loss_workspace(c.logits)))
    R.close(logprob, want, err + U * want.abs(), "logprob")


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("rows,vocab,dtype", [
    (128, 16_392, BF16), (130, 20_003, BF16), (129, 32_768, BF16), (131, 10_001, FP32),           # rows that 512 lanes hold by 8 words
    (128, 32_776, BF16), (130, 50_257, BF16), (130, 30_001, FP32),                                # by 16
    (128, 65_544, BF16), (260, 70_001, BF16), (300, 40_003, FP32), (511, 32_773, FP32),           # that 1024 lanes hold
])
def test_the_policy_loss_of_rows_that_a_workgroup_holds(rows, vocab, dtype, grad, tight):
    policy(Case(rows, vocab, dtype, temperature=0.9, pad=vocab % 3, shift=vocab % 5, masked=0.2, seed=52), grad=grad)
    if grad:
        policy(Case(rows, vocab, dtype, masked=0.2, seed=53), old=False, kl=None, in_place=True)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("temperature", [1e20, 1e30, 1e36, 1e38])
@pytest.mark.parametrize("rows,vocab", [(4, 40), (4, 70_001)])
def test_extreme_temperatures(rows, vocab, temperature, dtype, tight):
    # they give even a mask of the type's lowest value a chance again
    c = Case(rows, vocab, dtype, temperature=temperature, masked=0, seed=56)
    c.logits[:, 7:vocab // 2] = torch.finfo(dtype).min
    c.logits[1, 9:vocab - 9] = float("-inf")
    c.tokens.remainder_(7)
    if temperature == 1e38:
        c.tokens[0] = 8
    check_logprob(c)
    policy(c, scale=1e30)


@pytest.mark.parametrize("temperature", [0.6, 0.7, 0.9, 1.0, 1.3])
@pytest.mark.parametrize("vocab", [40, 3001])
def test_the_gradient_from_an_lse(vocab, temperature):
    # logits far from 0: what FP32 has lost of lse is all that the probabilities may be off by, beside roundings of the exponent itself.  With t = |x / T - lse|:
    # the difference, the factor and the exponent u t each, the power 2 u, the slope by T, its product and the result 3 u, the forward call's lse as above
    levels = torch.tensor([0.0, 30.0, -700.0, 1000.0, 5000.0, 20000.0, -60000.0])
    c = Case(len(levels), vocab, FP32, temperature=temperature, masked=0, seed=54)
    c.logits += levels.cuda()[:, None]
    lse = forward(c)[1]
    d = torch.full_like(c.logits, 7.0)
    fo.token_logprob_backward(c.logits, c.tokens, lse, torch.ones(c.rows, device="cuda"), d, temperature=temperature)
    t = float(torch.tensor(temperature, dtype=torch.float32))
    x = c.logits.double().cpu() / t
    want_lse = torch.logsumexp(x, 1, keepdim=True)
    p = torch.exp(x - want_lse)
    far = (p * (x.amax(1, keepdim=True) - x)).sum(1, keepdim=True)
    e = U * (want_lse.abs() + 3 * (x - want_lse).abs() + 5 + 2 * far + ADDS)
    err = p / t * (e + e * e)
    hit = torch.zeros_like(x).scatter_(1, c.tokens.cpu()[:, None], 1.0)
    R.close(d, (hit - p) / t, err + 3 * U * hit / t, "dlogits")


@pytest.mark.parametrize("temperature", [1e-30, 1e20, 1e27, 1e38])
def test_the_gradient_from_an_lse_at_extreme_temperatures(temperature):
    # beside a mask of the type's lowest value, which such temperatures give a chance again; the exponent's roundings are of values that may be as far apart
    c = Case(4, 300, FP32, temperature=temperature, masked=0, seed=55)
    if temperature < 1:
        c.logits *= temperature
    c.logits[:, 7:90] = torch.finfo(FP32).min
    lse = forward(c)[1]
    d = torch.full_like(c.logits, 7.0)
    fo.token_logprob_backward(c.logits, c.tokens, lse, torch.full((4,), min(temperature, 1e30), device="cuda"), d, temperature=temperature)
    t = float(torch.tensor(temperature, dtype=torch.float32))
    slope = float(torch.tensor(min(temperature, 1e30), dtype=torch.float32)) / t
    x = c.logits.double().cpu() / t
    want_lse = torch.logsumexp(x, 1, keepdim=True)
    p = torch.exp(x - want_lse)
    hit = torch.zeros_like(x).scatter_(1, c.tokens.cpu()[:, None], 1.0)
    far = (p * (x.amax(1, keepdim=True) - x)).sum(1, keepdim=True)
    e = U * (3 * want_lse.abs() + 3 * (x - want_lse).abs() + 5 + 2 * far + ADDS)
    R.close(d, (hit - p) * slope, slope * (p * (e + e * e) + 3 * U * hit) + 2.0 ** -148, "dlogits")
