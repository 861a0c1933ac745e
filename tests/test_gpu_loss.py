"""The losses on the logits and their gradients on the GPU, against their definitions in 64 bits (tests/loss_reference.py, where the
tolerances are derived)."""
import gc
import zlib

import pytest
import torch

import loss_reference as R
import paper_2602_23349_amd as fo

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
VOCABS = [1, 2, 7, 8, 9, 63, 64, 100, 1000, 1001, 2047, 2048, 2056, 4099, 8192, 8193, 16391, 32000, 50257, 65536, 65544, 128256, 131073, 262147]


@pytest.fixture(autouse=True)
def nothing_left_to_collect():
    gc.collect()


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


class Case:
    """Logits in rows `pad` values longer than the vocabulary that begin `shift` values behind an aligned address."""

    def __init__(self, rows, vocab, dtype=BF16, temperature=1.0, pad=0, shift=0, masked=0.25, seed=0, spread=3.0):
        g = gen(rows, vocab, str(dtype), seed)
        self.rows, self.vocab, self.dtype, self.temperature = rows, vocab, dtype, temperature
        values = torch.randn(rows, vocab, generator=g) * spread
        values[torch.arange(rows), torch.randint(0, vocab, (rows,), generator=g)] += 6 * torch.rand(rows, generator=g)
        self.logits = self.place(values, pad, shift)
        tokens = torch.randint(0, vocab, (rows,), generator=g)
        tokens[torch.rand(rows, generator=g) < masked] = -100
        self.tokens = tokens.cuda()
        vec = lambda s: (torch.randn(rows, generator=g) * s)        # noqa: E731
        self.advantages, self.near, self.far = vec(1.0).cuda(), vec(0.2), vec(0.3)
        w = torch.rand(rows, generator=g) + 0.1
        w[torch.rand(rows, generator=g) < 0.2] = 0
        self.weights = (w / rows).cuda()
        self.pad, self.shift = pad, shift

    def place(self, values, pad, shift):
        rows, vocab = values.shape
        flat = torch.full((rows * (vocab + pad) + shift,), 77.0, dtype=self.dtype, device="cuda")
        m = flat[shift:].view(rows, vocab + pad)[:, :vocab]
        m.copy_(values)
        self.flat = flat
        return m

    def room(self):
        """Memory for a gradient of the same layout, and a check that nothing but the matrix has been written."""
        flat = torch.full_like(self.flat, 55.0)
        m = flat[self.shift:].view(self.rows, self.vocab + self.pad)[:, :self.vocab]

        def untouched():
            rest = flat.clone()
            rest[self.shift:].view(self.rows, self.vocab + self.pad)[:, :self.vocab] = 55.0
            assert bool((rest == 55.0).all())
        return m, untouched


def memory(size):
    return torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if size else None


def forward(c, stream=None, workspace=None):
    logprob, lse = (torch.full((c.rows,), 7.0, device="cuda") for _ in range(2))
    if workspace is None:
        workspace = memory(fo.token_logprob_workspace(c.logits))
    fo.token_logprob(c.logits, c.tokens, logprob, lse, temperature=c.temperature, workspace=workspace, stream=stream)
    return logprob, lse


def check_logprob(c):
    logprob, lse = forward(c)
    ref = R.Rows(c.logits, c.tokens, c.temperature)
    wide = torch.full((c.rows,), 7.0, dtype=torch.float64, device="cuda")
    fo.token_logprob(c.logits, c.tokens, logprob64=wide, temperature=c.temperature, workspace=memory(fo.token_logprob_workspace(c.logits)))
    assert torch.equal(wide.float().nan_to_num(nan=-1.0), logprob.nan_to_num(nan=-1.0))
    R.close(wide, ref.logprob, torch.where(ref.counted, ref.err, 0.0) + 1e-14 * ref.logprob.abs(), "logprob64")
    R.close(logprob, ref.logprob, torch.where(ref.counted, ref.err, 0.0) + R.U * ref.logprob.abs(), "logprob")
    R.close(lse, ref.lse, torch.where(ref.counted, ref.err, 0.0) + R.U * ref.lse.abs(), "lse")
    return ref, lse


def check_backward(c, ref, lse, in_place=False):
    d = c.advantages.clone()
    d[::5] = 0
    out, untouched = c.room()
    target = c.logits if in_place else out
    fo.token_logprob_backward(c.logits, c.tokens, lse, d, target, temperature=c.temperature)
    want, err = ref.gradient(d.double().cpu(), torch.zeros(c.rows, dtype=torch.float64), True)
    R.close(target, want, err, "dlogits")
    if not in_place:
        untouched()


def policy(c, old=True, kl=0.05, low=0.2, high=0.28, weights=True, grad=True, in_place=False, scale=1.0, stream=None, workspace=None):
    ref = R.Rows(c.logits, c.tokens, c.temperature)
    lp = torch.nan_to_num(ref.logprob, nan=-1.0, neginf=-30.0).clamp(min=-60).float()
    # (no ratio so near a border that an FP32 sum could put it on the other side)
    close_by = ((torch.exp(-c.near) - 1 - high).abs() < 1e-3) | ((torch.exp(-c.near) - 1 + low).abs() < 1e-3)
    c.old = (lp + c.near + 0.01 * close_by).cuda() if old else None
    c.ref = (lp + c.far).cuda() if kl is not None else None
    c.spec = fo.PolicyLoss(clip_low=low, clip_high=high, kl_weight=kl or 0.0, temperature=c.temperature, grad_scale=scale)
    w = c.weights if weights else None
    want = R.Policy(ref, c.advantages, c.old, c.ref, w, low, high, kl or 0.0, scale)
    border = torch.stack([(want.ratio - 1 - high).abs(), (want.ratio - 1 + low).abs()]).nan_to_num(nan=1.0).amin(0)
    assert not old or bool((border > 20 * ref.err * want.ratio.nan_to_num(nan=0.0)).all())
    stats, logprob = torch.full((4,), 7.0, device="cuda"), torch.full((c.rows,), 7.0, device="cuda")
    out, untouched = c.room()
    target = None if not grad else c.logits if in_place else out
    if workspace is None:
        workspace = memory(fo.policy_loss_workspace(c.logits))
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    fo.policy_loss(c.spec, c.logits, c.tokens, c.advantages, stats, old_logprob=c.old, ref_logprob=c.ref, weights=w, logprob=logprob,
                   dlogits=target, workspace=workspace, stream=stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    R.close(stats, want.stats, want.stats_err, "stats")
    R.close(logprob, want.logprob, want.logprob_err, "logprob")
    if grad:
        dx, err = ref.gradient(want.slope, want.slope_err, False)
        R.close(target, dx, err, "dlogits")
    if not in_place:
        untouched()
    return stats, logprob, target


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_log_probabilities_and_their_gradient(vocab, dtype):
    c = Case(5, vocab, dtype, temperature=0.7 if vocab % 2 else 1.0)
    ref, lse = check_logprob(c)
    check_backward(c, ref, lse)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows", [1, 2, 63, 300, 1100])
def test_numbers_of_rows(rows, dtype):
    for vocab in (40, 5003):
        c = Case(rows, vocab, dtype)
        ref, lse = check_logprob(c)
        check_backward(c, ref, lse, in_place=True)
        policy(Case(rows, vocab, dtype, seed=1))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("words", [1, 512, 1024, 2048])
def test_log_probabilities_by_the_length_of_rows(words, dtype):
    # rows of as many words and of a few values less and more, by one wavefront to sixteen, in calls of few rows and of many
    size = 8 if dtype == BF16 else 4
    for rows in (2, 511, 512):
        for more in (-1, 0, 1, size + 1):
            c = Case(rows, words * size + more, dtype, pad=more % 4, seed=21)
            ref, lse = check_logprob(c)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("pad,shift", [(1, 0), (3, 1), (8, 8), (0, 3), (5, 7)])
def test_rows_at_any_address(pad, shift, dtype):
    for vocab in (3, 77, 2051, 20001):
        c = Case(4, vocab, dtype, pad=pad, shift=shift)
        ref, lse = check_logprob(c)
        check_backward(c, ref, lse)
        policy(Case(4, vocab, dtype, pad=pad, shift=shift, seed=2))
        policy(Case(4, vocab, dtype, pad=pad, shift=shift, seed=2), in_place=True)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_policy_loss_over_vocabularies(vocab, dtype):
    policy(Case(5, vocab, dtype, temperature=1.3 if vocab % 2 else 1.0, seed=3))
    policy(Case(5, vocab, dtype, seed=4), in_place=True)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17])
def test_policy_loss_of_a_few_rows(rows, dtype):
    # by one workgroup or several, at the lengths of rows where that changes
    for vocab in (1, 31, 2047, 2048, 2055, 4095, 4096, 4103):
        for old, kl in ((True, 0.1), (False, None)):
            policy(Case(rows, vocab, dtype, pad=vocab % 3, seed=20), old=old, kl=kl, weights=kl is None)


@pytest.mark.parametrize("old", [False, True])
@pytest.mark.parametrize("kl", [None, 0.0, 0.1])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("rows", [7, 700])
def test_policy_loss_options(old, kl, weights, rows):
    for grad in (False, True):
        policy(Case(rows, 333, BF16, seed=5), old=old, kl=kl, weights=weights, grad=grad, scale=-3.0)


def test_policy_loss_borders_are_inside():
    # the ratio of the policy to itself is 1 exactly, which a clip of 0 on either side does not block
    c = Case(40, 100, FP32, masked=0, seed=6)
    stats, _, d = policy(c, old=False, kl=None, low=0.0, high=0.0, weights=False)
    assert float(stats[3]) == 0 and bool((d != 0).any(1).all())
    # nothing is blocked above without an upper limit
    stats, _, _ = policy(Case(40, 100, FP32, masked=0, seed=6), kl=None, low=0.999, high=float("inf"), weights=False)
    assert float(stats[3]) == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("vocab", [9, 1000, 40003])
def test_masked_vocabularies(vocab, dtype):
    # tokens that are masked out by -infinity or the type's lowest value, all but one of a row's among them
    for low in (float("-inf"), torch.finfo(dtype).min):
        for keep in ("half", "one", "first", "last"):
            c = Case(6, vocab, dtype, temperature=0.8, masked=0, seed=7)
            g = gen(vocab, keep)
            there = {"half": torch.rand(6, vocab, generator=g) < 0.5, "one": torch.zeros(6, vocab, dtype=torch.bool),
                     "first": (torch.arange(vocab) == 0).expand(6, vocab).clone(), "last": (torch.arange(vocab) == vocab - 1).expand(6, vocab).clone()}[keep]
            tokens = c.tokens.cpu()
            if keep in ("half", "one"):
                there[torch.arange(6), tokens] = True
            else:
                tokens = torch.full((6,), 0 if keep == "first" else vocab - 1)
            c.tokens = tokens.cuda()
            c.logits.masked_fill_(~there.cuda(), low)
            ref, lse = check_logprob(c)
            check_backward(c, ref, lse)
            policy(c)
    # a row whose mask leaves nothing: by the lowest value all tokens are as likely as each other
    c = Case(3, vocab, dtype, masked=0, seed=8)
    c.logits.fill_(torch.finfo(dtype).min)
    check_logprob(c)
    policy(c, old=False, kl=None)


@pytest.mark.parametrize("vocab", [5, 1000, 70001])
def test_rows_without_a_result(vocab):
    c = Case(6, vocab, BF16, masked=0, seed=9)
    c.logits[0] = float("-inf")                       # nothing is left
    c.logits[1, vocab // 2] = float("nan")
    c.logits[2, vocab - 1] = float("inf")
    c.tokens[3] = vocab                               # no such token
    c.tokens[4] = 1 << 40
    logprob, lse = forward(c)
    assert bool(torch.isnan(logprob[:5]).all()) and not bool(torch.isnan(logprob[5]))
    assert float(lse[0]) == float("-inf") and bool(torch.isnan(lse[1:3]).all()) and bool(torch.isfinite(lse[3:]).all())
    d = torch.empty_like(c.logits)
    fo.token_logprob_backward(c.logits, c.tokens, lse, torch.ones(6, device="cuda"), d)
    assert bool(torch.isnan(d[:5]).all()) and bool(torch.isfinite(d[5]).all())
    # such rows do not reach the loss where they do not count, by their token or their weight
    for by_token in (True, False):
        tokens, w = c.tokens.clone(), torch.ones(6, device="cuda")
        if by_token:
            tokens[:5] = -1
        else:
            w[:5] = 0
        stats = torch.empty(4, device="cuda")
        d.fill_(7.0)
        a = torch.full((6,), float("nan"), device="cuda")
        a[5] = 1.0
        fo.policy_loss(fo.PolicyLoss(), c.logits, tokens, a, stats, weights=w, logprob=logprob, dlogits=d,
                       workspace=memory(fo.policy_loss_workspace(c.logits)))
        assert bool(torch.isfinite(stats).all()) and bool((d[:5] == 0).all()) and bool((d[5] != 0).any()) and bool((logprob[:5] == 0).all())
    # and where they do, the loss and their gradients say so
    fo.policy_loss(fo.PolicyLoss(), c.logits, c.tokens, torch.ones(6, device="cuda"), stats, logprob=logprob, dlogits=d,
                   workspace=memory(fo.policy_loss_workspace(c.logits)))
    assert bool(torch.isnan(stats[0])) and bool(torch.isnan(d[:5]).all()) and bool(torch.isfinite(d[5]).all())


@pytest.mark.parametrize("vocab", [9, 1000, 40003])
def test_a_token_of_probability_zero(vocab):
    c = Case(4, vocab, BF16, masked=0, seed=17)
    c.logits[1, c.tokens[1]] = float("-inf")
    a, stats, lp, d = torch.full((4,), 2.0, device="cuda"), torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(c.logits)
    call = lambda **kw: fo.policy_loss(fo.PolicyLoss(kl_weight=0.1), c.logits, c.tokens, a, stats, logprob=lp, dlogits=d,       # noqa: E731
                                       workspace=memory(fo.policy_loss_workspace(c.logits)), **kw)
    # the ratio of the policy to itself is 1 all the same
    call()
    ref = R.Rows(c.logits, c.tokens)
    want, err = ref.gradient(torch.full((4,), -2.0, dtype=torch.float64), torch.zeros(4, dtype=torch.float64), False)
    R.close(d, want, err, "dlogits")
    assert stats.tolist() == [-8.0, -8.0, 0.0, 0.0] and float(lp[1]) == float("-inf")
    # that to another policy is 0, and to a reference that gives it a chance the KL term is infinite
    call(old_logprob=torch.full((4,), -3.0, device="cuda"))
    assert bool((d[1] == 0).all()) and bool(torch.isfinite(stats).all())
    call(ref_logprob=torch.full((4,), -3.0, device="cuda"))
    assert float(stats[0]) == float("inf") and float(stats[2]) == float("inf") and float(stats[1]) == -8.0


@pytest.mark.parametrize("vocab", [9, 1000, 40003])
def test_the_gradient_from_an_lse_without_digits(vocab):
    # nothing but the type's lowest value: in FP32 lse does not differ from it by the vocabulary's size any more
    for low, dtype in ((torch.finfo(BF16).min, BF16), (torch.finfo(FP32).min, FP32), (-131072.0, FP32), (131072.0, BF16)):
        c = Case(3, vocab, dtype, masked=0, seed=18)
        c.logits[1] = low
        d, slopes = torch.empty_like(c.logits), torch.ones(3, device="cuda")
        lse = forward(c)[1]
        fo.token_logprob_backward(c.logits, c.tokens, lse, slopes, d)
        gone = bool(lse[1].abs() >= 131072)
        assert bool(torch.isfinite(d[::2]).all()) and bool(torch.isnan(d[1]).all()) == gone and (gone or low == -131072.0)
        slopes[1] = 0
        fo.token_logprob_backward(c.logits, c.tokens, lse, slopes, d)
        assert bool((d[1] == 0).all())


def test_preference_gradient_over_the_log_probabilities():
    for lengths in ([700, 300], [5, 9] * 20, [0, 4, 3000, 1]):
        lp, ref, w, cut = preference_case(lengths, 4, behind=3, ahead=2)
        lp, ref, w, cut = lp.cuda(), ref.cuda(), w.cuda(), cut.cuda()
        out, d = [torch.empty(1, device="cuda") for _ in range(2)], torch.empty_like(lp)
        fo.preference_loss(fo.PreferenceLoss(), lp, cut, out[0], ref_logprob=ref, weights=w, dlogprob=d)
        fo.preference_loss(fo.PreferenceLoss(), lp, cut, out[1], ref_logprob=ref, weights=w, dlogprob=lp)
        assert torch.equal(lp, d) and torch.equal(out[0], out[1])


@pytest.mark.parametrize("vocab", [11, 3001])
def test_gradients_against_differences(vocab):
    # the directional derivative of the loss, from two FP64 evaluations of its definition
    c = Case(3, vocab, FP32, temperature=0.9, masked=0, seed=10, spread=1.0)
    stats, _, d = policy(c, kl=0.2, weights=False)
    g = gen(vocab)
    direction = torch.randn(3, vocab, generator=g, dtype=torch.float64)
    x, h = c.logits.double().cpu(), 1e-5
    loss = [R.Policy(R.Rows(x + s * h * direction, c.tokens, 0.9), c.advantages, c.old, c.ref, None, 0.2, 0.28, 0.2).stats[0] for s in (1, -1)]
    slope = float((loss[0] - loss[1]) / (2 * h))
    got = float((d.double().cpu() * direction).sum())
    # differences: h^2 of the third derivative (the slopes and their sums are of order 10 here), and 1e-16 / h of the loss
    assert abs(got - slope) <= 1e-7 * vocab + 1e-5 * abs(slope) + 1e-4


def test_no_rows():
    x = torch.empty(0, 50, dtype=BF16, device="cuda")
    t, v = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    fo.token_logprob(x, t, v, v)
    fo.token_logprob_backward(x, t, v, v, x)
    stats = torch.full((4,), 7.0, device="cuda")
    fo.policy_loss(fo.PolicyLoss(), x, t, v, stats, dlogits=x)
    assert bool((stats == 0).all())


# ---------------------------------------------------------------------------------------- preference loss --

def preference_case(lengths, seed, masked=0.2, behind=0, ahead=0):
    g = gen(str(lengths), seed)
    n = sum(lengths)
    rows = ahead + n + behind
    cut = [ahead]
    for v in lengths:
        cut.append(cut[-1] + v)
    w = torch.rand(rows, generator=g)
    w[torch.rand(rows, generator=g) < masked] = 0
    lp = -torch.rand(rows, generator=g) * 5
    return lp, lp + 0.5 * torch.randn(rows, generator=g), w, torch.tensor(cut, dtype=torch.int64)


@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.1), ("sigmoid", 0.5), ("hinge", 0.0), ("squared", 0.0)])
@pytest.mark.parametrize("lengths", [[1, 1], [0, 3], [5, 0], [0, 0], [64, 65, 1, 1023], [2048, 3000], [7] * 34, [0, 1] * 70 + [300, 5]])
def test_preference_loss(kind, smoothing, lengths):
    for halves in (False, True):
        for given in (True, False):
            lp, ref, w, cut = preference_case(lengths, 1, behind=9 if halves else 0, ahead=4 if halves else 0)
            if not given:
                ref = w = None
            loss, margins, grad = R.preference(lp, cut, ref, w, kind, 0.3, smoothing, halves, 2.0)
            spec = fo.PreferenceLoss(beta=0.3, kind=kind, label_smoothing=smoothing, order="halves" if halves else "by_turns", grad_scale=2.0)
            cuda = lambda v: None if v is None else v.cuda()        # noqa: E731
            out, m, d = torch.full((1,), 7.0, device="cuda"), torch.full((len(lengths) // 2,), 7.0, device="cuda"), torch.full((lp.numel(),), 7.0, device="cuda")
            fo.preference_loss(spec, lp.cuda(), cut.cuda(), out, ref_logprob=cuda(ref), weights=cuda(w), margins=m, dlogprob=d)
            # sums are FP64: the results are off by their rounding to FP32 (and by what 10^4 additions in FP64 make of 10^4 values of up to 5)
            R.close(out, torch.tensor([loss]), torch.tensor([R.U * abs(loss) + 1e-9 * (1 + abs(loss))]), "loss")
            R.close(m, margins, R.U * margins.abs() + 1e-10, "margins")
            R.close(d, grad, R.U * grad.abs() + 1e-9 * (1 + grad.abs()), "dlogprob")
            again = [t.clone() for t in (out, m, d)]
            fo.preference_loss(spec, lp.double().cuda(), cut.cuda(), out, ref_logprob=cuda(ref), weights=cuda(w), margins=m, dlogprob=d)
            assert all(torch.equal(a, b) for a, b in zip(again, (out, m, d)))


def test_preference_loss_of_values_that_do_not_count():
    lp, ref, w, cut = preference_case([6, 6], 2, masked=0.0)
    lp[2], lp[8], w[2], w[8] = float("nan"), float("-inf"), 0, 0
    loss, margins, grad = R.preference(torch.nan_to_num(lp, neginf=0.0), cut, ref, w)
    out, m, d = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(12, device="cuda")
    fo.preference_loss(fo.PreferenceLoss(), lp.cuda(), cut.cuda(), out, ref_logprob=ref.cuda(), weights=w.cuda(), margins=m, dlogprob=d)
    assert abs(float(out) - loss) < 1e-6 and bool(torch.isfinite(d).all()) and float(d[2]) == 0 and float(d[8]) == 0
    # infinitely far apart: no loss and no slope in one direction, an infinite loss in the other
    for kind, sign in (("sigmoid", 1), ("hinge", 1), ("sigmoid", -1), ("hinge", -1)):
        lp = torch.zeros(2)
        lp[1 if sign > 0 else 0] = float("-inf")
        fo.preference_loss(fo.PreferenceLoss(kind=kind), lp.cuda(), torch.tensor([0, 1, 2]).cuda(), out, margins=m)
        assert float(out) == (0.0 if sign > 0 else float("inf")) and float(m) == sign * float("inf")
    # no pairs, and bounds outside the rows
    fo.preference_loss(fo.PreferenceLoss(), lp.cuda(), torch.tensor([0]).cuda(), out, dlogprob=d[:2])
    assert float(out) == 0 and bool((d[:2] == 0).all())
    lp, _, _, _ = preference_case([3, 3], 3)
    want = R.preference(lp, [0, 3, 6])
    fo.preference_loss(fo.PreferenceLoss(), lp.cuda(), torch.tensor([-5, 3, 1 << 60]).cuda(), out, margins=m, dlogprob=d[:6])
    assert abs(float(out) - want[0]) < 1e-6 and abs(float(m) - float(want[1])) < 1e-6


# -------------------------------------------------------------------------------- together, streams, graphs --

def whole(x, tokens, cut, ref, w, out):
    """Log-probabilities, preference loss and the gradient of the logits, as a training step calls them."""
    fo.token_logprob(x, tokens, out["lp"], out["lse"], workspace=out["ws"])
    fo.preference_loss(out["spec"], out["lp"], cut, out["loss"], ref_logprob=ref, weights=w, margins=out["m"], dlogprob=out["d"])
    fo.token_logprob_backward(x, tokens, out["lse"], out["d"], out["dx"])


def room_for(x, pairs):
    rows = x.shape[0]
    v = lambda n: torch.full((n,), 7.0, device="cuda")        # noqa: E731
    return dict(spec=fo.PreferenceLoss(beta=0.2), lp=v(rows), lse=v(rows), loss=v(1), m=v(pairs), d=v(rows), dx=torch.full_like(x, 7.0),
                ws=memory(fo.token_logprob_workspace(x)))


def test_preference_step_matches_autograd():
    c = Case(90, 517, FP32, masked=0.3, seed=11)
    cut = torch.tensor([0, 20, 45, 45, 90])
    ref = torch.randn(90, generator=gen(1)) - 6
    w = (c.tokens >= 0).float()
    out = room_for(c.logits, 2)
    whole(c.logits, c.tokens, cut.cuda(), ref.cuda(), w, out)
    x = c.logits.double().cpu().requires_grad_()
    lp = torch.log_softmax(x, 1).gather(1, c.tokens.cpu().clamp(min=0)[:, None])[:, 0]
    gap = w.cpu() * (lp - ref)
    z = 0.2 * torch.stack([gap[0:20].sum() - gap[20:45].sum(), gap[45:45].sum() - gap[45:90].sum()])
    loss = torch.nn.functional.softplus(-z).mean()
    loss.backward()
    assert abs(float(out["loss"]) - loss.item()) <= 1e-5 * loss.item()
    # log-probabilities are off by a few u of 10 each, the gradient's scale by that of 70 of them
    assert float((out["dx"].double().cpu() - x.grad).abs().max()) <= 1e-5 * float(x.grad.abs().max())


def test_results_are_the_same_bits_every_time_and_on_any_stream():
    c = Case(300, 5003, BF16, seed=12)
    first = [t.clone() for t in policy(c)]
    side = torch.cuda.Stream()
    for stream in (side, None, side):
        again = policy(c, stream=stream)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("rows,vocab,dtype", [(3, 2001, FP32), (700, 1003, BF16), (2, 131080, BF16), (260, 70001, BF16)])
def test_captured_losses_replay_like_eager_calls(rows, vocab, dtype):
    c, other = Case(rows, vocab, dtype, seed=13), Case(rows, vocab, dtype, seed=14)
    cut = torch.tensor([0, rows // 2, rows]).cuda()
    ref = torch.randn(rows, generator=gen(2)).cuda() - 8
    x, tokens = c.logits.clone(), c.tokens.clone()
    spec = fo.PolicyLoss(kl_weight=0.1)

    def both(x, tokens, out, p):
        whole(x, tokens, cut, ref, None, out)
        fo.policy_loss(spec, x, tokens, c.advantages, p["stats"], ref_logprob=ref, weights=c.weights, logprob=p["lp"], dlogits=p["dx"],
                       workspace=p["ws"])

    def room():
        return room_for(x, 1), dict(stats=torch.empty(4, device="cuda"), lp=torch.empty(rows, device="cuda"), dx=torch.empty_like(x),
                                    ws=memory(fo.policy_loss_workspace(x)))
    got, want = room(), room()
    both(x, tokens, *got)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(x, tokens, *got)
    for replay in range(4):
        src = (c, other)[replay % 2]
        x.copy_(src.logits)
        tokens.copy_(src.tokens)
        for v in (got[0]["lp"], got[0]["d"], got[1]["stats"], got[1]["dx"], got[0]["dx"]):
            v.fill_(7.0)
        graph.replay()
        both(src.logits, src.tokens, *want)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            for k in a:
                if k not in ("spec", "ws"):
                    assert torch.equal(a[k].nan_to_num(nan=-5.0), b[k].nan_to_num(nan=-5.0)), (replay, k)


def test_two_calls_at_once():
    # on two streams, each with its own workspace
    cases = [Case(64, 40001, BF16, seed=s) for s in (15, 16)]
    want = [[t.clone() for t in policy(c)] for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    outs = []
    for c in cases:
        outs.append(dict(stats=torch.empty(4, device="cuda"), lp=torch.empty(64, device="cuda"), dx=torch.empty_like(c.logits),
                         ws=memory(fo.policy_loss_workspace(c.logits))))
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s, o in zip(cases, streams, outs):
            fo.policy_loss(c.spec, c.logits, c.tokens, c.advantages, o["stats"], old_logprob=c.old, ref_logprob=c.ref, weights=c.weights,
                           logprob=o["lp"], dlogits=o["dx"], workspace=o["ws"], stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(a, b) for a, b in zip(w, (o["stats"], o["lp"], o["dx"])))


def test_offsets_beyond_32_bits():
    # a gradient of more than 2^31 values, and rows whose bytes begin beyond 2^32
    rows, vocab = 17000, 131072
    x = torch.zeros(rows, vocab, dtype=BF16, device="cuda")
    at = [0, 8191, 16384, rows - 1]
    g = gen(3)
    for r in at:
        x[r] = torch.randn(vocab, generator=g).cuda()
    tokens = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    tokens[at] = torch.tensor([0, 5, vocab - 1, 77], device="cuda")
    stats, lp = torch.empty(4, device="cuda"), torch.empty(rows, device="cuda")
    a = torch.ones(rows, device="cuda")
    ws = memory(fo.policy_loss_workspace(x))
    fo.policy_loss(fo.PolicyLoss(), x, tokens, a, stats, logprob=lp, dlogits=x, workspace=ws)
    assert abs(float(stats[0]) + 4) < 1e-6
    for r in at:
        assert abs(float(x[r].double().sum())) < 0.05 and float(x[r, tokens[r]]) < -0.9
    assert int(torch.count_nonzero(x)) <= 4 * vocab and float(lp[1]) == 0
