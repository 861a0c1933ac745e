"""Lists of gradients that follow a list of parameters, without a GPU: what a call is given is looked at instead of the call itself."""
import ctypes as C
import types

import pytest
import torch
from torch._subclasses import FakeTensorMode

import paper_2602_23349_amd as fo
from paper_2602_23349_amd import _marshal as M
from paper_2602_23349_amd import binding as B


class Tensor:
    """What the binding looks at of a tensor, on a GPU that exists in name only."""
    dtype = torch.bfloat16

    def __init__(self, address, device=0):
        self.data_ptr, self.get_device, self.is_cuda = lambda: address, lambda: device, device >= 0


class Factor:
    address = 0x10000

    def __init__(self, device=0):
        self.device = device


def parameters(*grads):
    fields = ("param", "rho", "m_q", "m_scale", "v_q", "v_scale")
    return fo.TensorList(types.SimpleNamespace(**{f: None for f in fields}, grad=g, numel=8 + i, lr=0.1, weight_decay=0.0) for i, g in enumerate(grads))


@pytest.fixture
def seen(monkeypatch):
    """The lists that the calls are given: (src, dst, numel) of each gradient."""
    lists = []

    def call(address, n, *rest):
        lists.append([(g.src, g.dst, g.numel) for g in (B._Gradient * n).from_address(address)])
        return 0
    monkeypatch.setattr(B, "_fast", types.SimpleNamespace(grad_norm=call, clip=call, follow=M.follow))
    return lists


def test_a_list_follows_the_gradients_of_its_parameters(seen):
    params = parameters(Tensor(0x1000), Tensor(0x2000), Tensor(0x3000))
    grads = fo.GradList.of(params)
    for changed in (None, 1, 0, 1):
        if changed is not None:
            params.set_grad(changed, Tensor(0x100000 * (len(seen) + 1)))
        fo.grad_norm(grads, 1.0, Factor())
        fo.clip_gradients(grads, Factor())
        now = [(t.grad, t.grad, t.numel) for t in params.array]
        assert seen[-2] == seen[-1] == now and now[2] == (0x3000, 0x3000, 10)
    # one that is taken away is refused by the call, which sees no address
    params.set_grad(2, None)
    fo.grad_norm(grads, 1.0, Factor())
    assert seen[-1][2] == (None, None, 10)


def test_a_list_of_tensors_stays_as_it_is(seen):
    class Whole(Tensor):
        is_contiguous, numel = (lambda self: True), (lambda self: 8)
    grads = fo.GradList([Whole(0x1000), Whole(0x2000)])
    fo.grad_norm(grads, 1.0, Factor())
    assert seen == [[(0x1000, 0x1000, 8), (0x2000, 0x2000, 8)]]


def test_parameters_on_another_device_than_the_factor_are_refused(seen):
    for grads in ((Tensor(0x1000, 1), Tensor(0x2000, 1)), (None, Tensor(0x2000, 1))):
        followed = fo.GradList.of(parameters(*grads))
        for call in (lambda: fo.grad_norm(followed, 1.0, Factor()), lambda: fo.clip_gradients(followed, Factor())):
            with pytest.raises(ValueError):
                call()
    for grads in ((Tensor(0x1000), Tensor(0x2000, 1)), (Tensor(0x1000, -1),)):
        with pytest.raises(ValueError):
            fo.GradList.of(parameters(*grads))
    # and where a gradient comes later: from another device, from the host, and back
    params = parameters(Tensor(0x1000), Tensor(0x2000), None)
    for of in (params, params.slice(1)):
        followed, last = fo.GradList.of(of), of.n - 1
        for device, good in ((0, True), (1, False), (0, True), (-1, False), (0, True)):
            of.set_grad(last, Tensor(0x4000, device))
            if good:
                fo.grad_norm(followed, 1.0, Factor())
                continue
            with pytest.raises(ValueError):
                fo.grad_norm(followed, 1.0, Factor())
    assert len(seen) == 6
    fo.grad_norm(fo.GradList.of(parameters()), 1.0, Factor(1))


STEPS = {"adamw_step": (0.9, 0.99, 1e-8, 1), "adamw_step_exact": (0.9, 0.99, 1e-8, 1), "sgd_step": (0.9,), "lion_step": (0.9, 0.99)}


def test_a_factor_on_another_device_than_the_current_one_is_refused(monkeypatch):
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append(name) or 0
    monkeypatch.setattr(B, "load_library", lambda: Library())
    monkeypatch.setattr(B, "_raw_current_device", lambda: 0)
    with pytest.raises(ValueError):
        fo.clip_factor_from_sum(Factor(1), 1.0, stream=0)
    fo.clip_factor_from_sum(Factor(0), 1.0, stream=0)
    here, there, mixed = (parameters(*[Tensor(0x1000 * (i + 1), d) for i, d in enumerate(on)]) for on in ((0, 0), (1, 1), (0, 1)))
    for name, hp in STEPS.items():
        step = getattr(fo, name)
        for tensors, factor in ((here, 1), (there, 1), (there, 0), (mixed, 0)):
            with pytest.raises(ValueError):
                step(tensors, *hp, stream=0, clip=Factor(factor))
        step(here, *hp, stream=0, clip=Factor(0))
        step(there, *hp, stream=0)                                   # without a factor the steps do not ask
    assert calls == ["flashoptim_clip_factor_from_sum"] + [f"flashoptim_{name}{end}" for name in STEPS for end in ("_clipped", "")]


@pytest.fixture
def marshal(monkeypatch):
    """The C++ module with the library's entry points, the current device being 0."""
    names = [n for n in B.EXPORTED_SYMBOLS if n.startswith(("flashoptim_mx4_", "flashoptim_block_norm", "flashoptim_token_logprob", "flashoptim_policy_loss",
                                                            "flashoptim_preference_loss", "flashoptim_grad_norm", "flashoptim_clip_gradients"))]
    M.bind({n: C.cast(getattr(fo.load_library(), n), C.c_void_p).value for n in names}, lambda device: 0, lambda: 0)
    monkeypatch.setattr(B, "_fast", M)
    monkeypatch.setattr(B, "_raw_current_device", lambda: 0)


class Stream:
    cuda_stream = 0

    def __init__(self, device):
        self.device_index = device


def test_another_device_is_refused_on_a_given_stream_too(marshal):
    class Whole(Tensor):
        is_contiguous, numel = (lambda self: True), (lambda self: 8)
    for device, streams in ((1, (0, Stream(0), Stream(1))), (0, (Stream(1),))):
        grads, factor = fo.GradList([Whole(0x1000, device)]), Factor(device)
        for stream in streams:
            with pytest.raises(ValueError, match="device"):
                fo.grad_norm(grads, 1.0, factor, stream=stream)
            with pytest.raises(ValueError, match="device"):
                fo.clip_gradients(grads, factor, stream=stream)
            with pytest.raises(ValueError, match="device"):
                fo.clip_factor_from_sum(factor, 1.0, stream=stream)
    with pytest.raises(ValueError, match="device"):
        fo.adamw_step(parameters(Tensor(0x1000)), 0.9, 0.99, 1e-8, 1, stream=Stream(1), clip=Factor(0))


@pytest.mark.filterwarnings("ignore")
def test_logits_on_another_device_are_refused(marshal):
    # tensors on GPUs that exist in name only: they are refused before anything asks for their memory
    policy, preference = fo.PolicyLoss(), fo.PreferenceLoss()
    with FakeTensorMode():
        def calls(x, tokens, vec, wide, cuts, stream):
            return [lambda: fo.token_logprob(x, tokens, vec, vec, stream=stream), lambda: fo.token_logprob(x, tokens, logprob64=wide, stream=stream),
                    lambda: fo.token_logprob_backward(x, tokens, vec, vec, x, stream=stream),
                    lambda: fo.policy_loss(policy, x, tokens, vec, vec, dlogits=x, stream=stream),
                    lambda: fo.preference_loss(preference, vec, cuts, vec[:1], stream=stream)]
        on = [(torch.empty(4, 64, dtype=torch.bfloat16, device=d), torch.zeros(4, dtype=torch.int64, device=d), torch.empty(4, device=d),
               torch.empty(4, dtype=torch.float64, device=d), torch.zeros(3, dtype=torch.int64, device=d)) for d in ("cuda:0", "cuda:1")]
        for tensors, streams in ((on[1], (None, 0, Stream(0), Stream(1))), (on[0], (Stream(1),))):
            for stream in streams:
                for call in calls(*tensors, stream):
                    with pytest.raises(ValueError, match="device"):
                        call()
        for k in range(5):
            mixed = [on[1 if i == k else 0][i] for i in range(5)]
            refused = 0
            for call in calls(*mixed, 0):
                try:
                    call()
                except ValueError as e:
                    refused += "device" in str(e)
                except Exception:                    # (no memory, where all lie on the current device)
                    pass
            assert refused == (4, 4, 4, 1, 1)[k], k
