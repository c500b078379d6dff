"""Host-side checks of the training-side entry points that need no GPU: refusals
of arguments, workspace sizes, records."""
import ctypes
import math

import pytest
import torch

import paper_2606_11660_gb300 as bg

FAKE = 0x7F0000000000  # aligned, never dereferenced: validation fails first or no device
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def built_library():
    from paper_2606_11660_gb300 import _build
    _build.build()
    yield


def accepted(st):
    """Past validation: without a device the pointers' lookup fails."""
    return st == bg.BERGSON_ECUDA


@pytest.fixture(autouse=True)
def no_launch():
    """What passes validation returns an injected status and enqueues nothing."""
    bg.bergson_debug_inject_status(bg.BERGSON_ECUDA, 1 << 20)
    yield
    bg.bergson_debug_inject_status(0, 0)


def fwd(**kw):
    a = dict(x=FAKE, dtype=bg.BERGSON_BF16, rows=4, V=100, ld=100, t=FAKE, tau=1.0, logp=FAKE,
             lse=FAKE, ent=FAKE)
    a.update(kw)
    return bg.lib().bergson_token_logprobs(*a.values(), None)


def bwd(**kw):
    a = dict(x=FAKE, dtype=bg.BERGSON_BF16, rows=4, V=100, ld=100, t=FAKE, tau=1.0, lse=FAKE,
             ent=FAKE, w=FAKE, h=FAKE, dx=FAKE + 4096, ld_d=100)
    a.update(kw)
    return bg.lib().bergson_token_logprobs_backward(*a.values(), None)


LOGITS_BAD = [
    (dict(dtype=3), bg.BERGSON_EINVAL), (dict(rows=-1), bg.BERGSON_EINVAL),
    (dict(rows=1 << 31), bg.BERGSON_EINVAL), (dict(V=0), bg.BERGSON_EINVAL),
    (dict(V=1 << 31, ld=1 << 31), bg.BERGSON_EINVAL), (dict(ld=99), bg.BERGSON_EINVAL),
    (dict(ld=1 << 41), bg.BERGSON_EUNSUPPORTED), (dict(x=None), bg.BERGSON_EINVAL),
    (dict(x=FAKE + 1), bg.BERGSON_EALIGN), (dict(dtype=0, x=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(t=None), bg.BERGSON_EINVAL), (dict(t=FAKE + 4), bg.BERGSON_EALIGN),
    (dict(tau=0.0), bg.BERGSON_EINVAL), (dict(tau=-1.0), bg.BERGSON_EINVAL),
    (dict(tau=NAN), bg.BERGSON_EINVAL), (dict(tau=INF), bg.BERGSON_EINVAL),
    (dict(tau=1e-50), bg.BERGSON_EINVAL), (dict(tau=1e60), bg.BERGSON_EINVAL),
    (dict(tau=3e-39), bg.BERGSON_EINVAL),
    (dict(lse=None), bg.BERGSON_EINVAL), (dict(lse=FAKE + 2), bg.BERGSON_EALIGN),
]


@pytest.mark.parametrize("kw,code", LOGITS_BAD + [
    (dict(logp=None), bg.BERGSON_EINVAL), (dict(logp=FAKE + 1), bg.BERGSON_EALIGN),
    (dict(ent=FAKE + 3), bg.BERGSON_EALIGN)])
def test_logprob_refusals(kw, code):
    assert fwd(**kw) == code and bg.bergson_last_error() != ""


@pytest.mark.parametrize("kw,code", LOGITS_BAD + [
    (dict(w=None, h=None), bg.BERGSON_EINVAL), (dict(ent=None), bg.BERGSON_EINVAL),
    (dict(dx=None), bg.BERGSON_EINVAL), (dict(dx=FAKE + 1), bg.BERGSON_EALIGN),
    (dict(ld_d=99), bg.BERGSON_EINVAL), (dict(dx=FAKE, ld_d=104), bg.BERGSON_EINVAL),
    (dict(w=FAKE + 2), bg.BERGSON_EALIGN), (dict(h=FAKE + 2), bg.BERGSON_EALIGN)])
def test_logprob_backward_refusals(kw, code):
    assert bwd(**kw) == code and bg.bergson_last_error() != ""


def test_logprob_calls_that_pass():
    for call in (fwd(), fwd(ent=None), fwd(x=FAKE + 2), fwd(ld=101), bwd(), bwd(h=None, ent=None),
                 bwd(w=None), bwd(dx=FAKE), fwd(rows=0, x=None, t=None, logp=None, lse=None)):
        assert accepted(call), bg.bergson_last_error()


def policy(ws=FAKE, ws_bytes=None, **kw):
    a = dict(logp=FAKE, old_logp=FAKE, ref_logp=FAKE, entropy=FAKE, advantages=FAKE, mask=FAKE,
             ld_logp=50, ld_old=50, ld_ref=50, ld_entropy=50, ld_adv=0, ld_mask=50, B=4, T=50,
             clip_low=0.2, clip_high=0.2, kl_coef=0.1, entropy_coef=0.1, norm_tokens=10.0, loss=FAKE,
             seq_loss=FAKE, stats=FAKE, d_logp=FAKE, d_entropy=FAKE, ld_d=50, ld_de=50,
             reduction=bg.BERGSON_POLICY_SUM_NORM, reserved=0)
    a.update(kw)
    n = 1 << 30 if ws_bytes is None else ws_bytes
    return bg.lib().bergson_policy_loss(bg.bergson_policy_args(**a), ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), bg.BERGSON_EINVAL), (dict(T=1 << 31), bg.BERGSON_EINVAL),
    (dict(B=1 << 20, T=1 << 21), bg.BERGSON_EUNSUPPORTED), (dict(reduction=3), bg.BERGSON_EINVAL),
    (dict(reserved=1), bg.BERGSON_EINVAL), (dict(clip_low=-0.1), bg.BERGSON_EINVAL),
    (dict(clip_low=1.1), bg.BERGSON_EINVAL), (dict(clip_high=-1.0), bg.BERGSON_EINVAL),
    (dict(clip_high=INF), bg.BERGSON_EINVAL), (dict(kl_coef=NAN), bg.BERGSON_EINVAL),
    (dict(entropy_coef=INF), bg.BERGSON_EINVAL), (dict(norm_tokens=0.0), bg.BERGSON_EINVAL),
    (dict(ref_logp=None), bg.BERGSON_EINVAL), (dict(entropy=None), bg.BERGSON_EINVAL),
    (dict(ld_adv=49), bg.BERGSON_EINVAL), (dict(ld_logp=49), bg.BERGSON_EINVAL),
    (dict(ld_old=0), bg.BERGSON_EINVAL), (dict(ld_ref=-1), bg.BERGSON_EINVAL),
    (dict(ld_entropy=49), bg.BERGSON_EINVAL), (dict(ld_mask=49), bg.BERGSON_EINVAL),
    (dict(ld_d=49), bg.BERGSON_EINVAL), (dict(ld_de=49), bg.BERGSON_EINVAL),
    (dict(logp=None), bg.BERGSON_EINVAL), (dict(old_logp=None), bg.BERGSON_EINVAL),
    (dict(advantages=None), bg.BERGSON_EINVAL), (dict(d_logp=None), bg.BERGSON_EINVAL),
    (dict(loss=None), bg.BERGSON_EINVAL), (dict(logp=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(stats=FAKE + 1), bg.BERGSON_EALIGN), (dict(seq_loss=FAKE + 1), bg.BERGSON_EALIGN),
    (dict(ws=None), bg.BERGSON_EINVAL), (dict(ws=FAKE + 16), bg.BERGSON_EALIGN),
    (dict(ws_bytes=16), bg.BERGSON_EWORKSPACE),
])
def test_policy_refusals(kw, code):
    assert policy(**kw) == code and bg.bergson_last_error() != ""


def test_policy_calls_that_pass():
    need = bg.bergson_policy_loss_workspace(4, 50)
    assert need > 0 and need % 256 == 0
    for st in (policy(), policy(ws_bytes=need), policy(mask=None, ld_mask=0), policy(mask=FAKE + 1),
               policy(kl_coef=0.0, ref_logp=None, ld_ref=0), policy(ld_adv=50),
               policy(entropy_coef=0.0, entropy=None, d_entropy=None, ld_de=0),
               policy(seq_loss=None, stats=None),
               policy(reduction=bg.BERGSON_POLICY_TOKEN_MEAN, norm_tokens=0.0),
               policy(B=0, logp=None, advantages=None), policy(T=0, logp=None)):
        assert accepted(st), bg.bergson_last_error()
    assert bg.lib().bergson_policy_loss(None, FAKE, 1 << 20, None) == bg.BERGSON_EINVAL
    assert bg.lib().bergson_policy_loss_workspace(4, 4, None) == bg.BERGSON_EINVAL
    with pytest.raises(bg.BergsonError):
        bg.bergson_policy_loss_workspace(-1, 4)


def preference(**kw):
    a = dict(logp=FAKE, ref_logp=FAKE, mask=FAKE, ld_logp=50, ld_ref=50, ld_mask=50, P=4, T=50,
             beta=0.1, margin=0.0, label_smoothing=0.1, loss=FAKE, pair_loss=FAKE, rewards=FAKE,
             d_logp=FAKE, ld_d=50, kind=0, mean_logp=0)
    a.update(kw)
    return bg.lib().bergson_preference_loss(bg.bergson_preference_args(**a), None)


@pytest.mark.parametrize("kw,code", [
    (dict(P=-1), bg.BERGSON_EINVAL), (dict(P=1 << 30), bg.BERGSON_EINVAL),
    (dict(T=-1), bg.BERGSON_EINVAL), (dict(P=1 << 25, T=1 << 20), bg.BERGSON_EUNSUPPORTED),
    (dict(kind=3), bg.BERGSON_EINVAL), (dict(beta=0.0), bg.BERGSON_EINVAL),
    (dict(beta=INF), bg.BERGSON_EINVAL), (dict(margin=NAN), bg.BERGSON_EINVAL),
    (dict(label_smoothing=1.5), bg.BERGSON_EINVAL), (dict(label_smoothing=NAN), bg.BERGSON_EINVAL),
    (dict(ld_logp=49), bg.BERGSON_EINVAL), (dict(ld_ref=49), bg.BERGSON_EINVAL),
    (dict(ld_mask=49), bg.BERGSON_EINVAL), (dict(ld_d=49), bg.BERGSON_EINVAL),
    (dict(logp=None), bg.BERGSON_EINVAL), (dict(pair_loss=None), bg.BERGSON_EINVAL),
    (dict(d_logp=None), bg.BERGSON_EINVAL), (dict(loss=None), bg.BERGSON_EINVAL),
    (dict(rewards=FAKE + 2), bg.BERGSON_EALIGN), (dict(ref_logp=FAKE + 1), bg.BERGSON_EALIGN),
])
def test_preference_refusals(kw, code):
    assert preference(**kw) == code and bg.bergson_last_error() != ""


def test_preference_calls_that_pass():
    for st in (preference(), preference(ref_logp=None, ld_ref=0, mask=None, ld_mask=0, rewards=None),
               preference(T=0, logp=None, d_logp=None), preference(P=0, logp=None, pair_loss=None),
               preference(label_smoothing=1.0)):
        assert accepted(st), bg.bergson_last_error()
    assert bg.lib().bergson_preference_loss(None, None) == bg.BERGSON_EINVAL


def adamw(lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, step=1, gs=None, n_tensors=1, **kw):
    a = dict(param=FAKE, grad=FAKE, master=FAKE, m=FAKE, v=FAKE, m_scale=FAKE, v_scale=FAKE, n=100,
             lr_scale=1.0, weight_decay=0.0, param_dtype=1, grad_dtype=1,
             state_kind=bg.BERGSON_STATE_8BIT, reserved=0)
    a.update(kw)
    arr = (bg.bergson_adamw_tensor * 1)(bg.bergson_adamw_tensor(**a))
    return bg.lib().bergson_adamw_step(arr, n_tensors, lr, b1, b2, eps, step, 0, gs, None)


@pytest.mark.parametrize("kw,code", [
    (dict(lr=NAN), bg.BERGSON_EINVAL), (dict(b1=1.0), bg.BERGSON_EINVAL),
    (dict(b2=-0.1), bg.BERGSON_EINVAL), (dict(b2=NAN), bg.BERGSON_EINVAL),
    (dict(eps=-1e-8), bg.BERGSON_EINVAL), (dict(step=0), bg.BERGSON_EINVAL),
    (dict(gs=FAKE + 2), bg.BERGSON_EALIGN), (dict(n_tensors=-1), bg.BERGSON_EINVAL),
    (dict(param_dtype=4), bg.BERGSON_EINVAL), (dict(grad_dtype=-1), bg.BERGSON_EINVAL),
    (dict(state_kind=2), bg.BERGSON_EINVAL), (dict(reserved=1), bg.BERGSON_EINVAL),
    (dict(n=-1), bg.BERGSON_EINVAL), (dict(n=1 << 39), bg.BERGSON_EUNSUPPORTED),
    (dict(lr_scale=NAN), bg.BERGSON_EINVAL), (dict(weight_decay=INF), bg.BERGSON_EINVAL),
    (dict(param=None), bg.BERGSON_EINVAL), (dict(grad=None), bg.BERGSON_EINVAL),
    (dict(m=None), bg.BERGSON_EINVAL), (dict(v=None), bg.BERGSON_EINVAL),
    (dict(m_scale=None), bg.BERGSON_EINVAL), (dict(v_scale=None), bg.BERGSON_EINVAL),
    (dict(param=FAKE + 1), bg.BERGSON_EALIGN), (dict(master=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(m_scale=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(state_kind=0, m=FAKE + 1), bg.BERGSON_EALIGN),
])
def test_adamw_refusals(kw, code):
    assert adamw(**kw) == code and bg.bergson_last_error() != ""


def test_adamw_calls_that_pass():
    for st in (adamw(), adamw(master=None), adamw(m=FAKE + 1, v=FAKE + 3), adamw(param=FAKE + 2),
               adamw(state_kind=0, m_scale=None, v_scale=None), adamw(n=0, param=None),
               adamw(step=1 << 40, eps=0.0, b1=0.0)):
        assert accepted(st), bg.bergson_last_error()
    assert bg.lib().bergson_adamw_step(None, 1, 1e-3, 0.9, 0.99, 1e-8, 1, 0, None,
                                       None) == bg.BERGSON_EINVAL


@pytest.mark.parametrize("args,code", [
    ((FAKE, FAKE, -1, 0, FAKE), bg.BERGSON_EINVAL), ((FAKE, FAKE, 1 << 39, 0, FAKE), bg.BERGSON_EUNSUPPORTED),
    ((FAKE, FAKE, 5, 2, FAKE), bg.BERGSON_EINVAL), ((None, FAKE, 5, 0, FAKE), bg.BERGSON_EINVAL),
    ((FAKE, None, 5, 0, FAKE), bg.BERGSON_EINVAL), ((FAKE, FAKE, 5, 1, FAKE + 1), bg.BERGSON_EALIGN),
    ((FAKE, FAKE + 2, 5, 1, FAKE), bg.BERGSON_EALIGN)])
def test_state_value_refusals(args, code):
    assert bg.lib().bergson_adamw_state_values(*args, None) == code


def moments(correction=1.0, floor=1e-12, ws=FAKE, ws_bytes=1 << 30, n_mats=1, **kw):
    a = dict(v=FAKE, v_scale=FAKE, d_out=100, d_in=60, r=FAKE, c=FAKE, state_kind=1, reserved=0)
    a.update(kw)
    arr = (bg.bergson_moment_matrix * 1)(bg.bergson_moment_matrix(**a))
    return bg.lib().bergson_factor_moments(arr, n_mats, correction, floor, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(correction=0.0), bg.BERGSON_EINVAL), (dict(correction=INF), bg.BERGSON_EINVAL),
    (dict(floor=0.0), bg.BERGSON_EINVAL), (dict(floor=1e-60), bg.BERGSON_EINVAL),
    (dict(floor=NAN), bg.BERGSON_EINVAL), (dict(d_out=0), bg.BERGSON_EINVAL),
    (dict(d_in=(1 << 24) + 1), bg.BERGSON_EINVAL),
    (dict(d_out=1 << 24, d_in=1 << 24), bg.BERGSON_EUNSUPPORTED),
    (dict(state_kind=5), bg.BERGSON_EINVAL), (dict(reserved=7), bg.BERGSON_EINVAL),
    (dict(v=None), bg.BERGSON_EINVAL), (dict(v_scale=None), bg.BERGSON_EINVAL),
    (dict(r=None), bg.BERGSON_EINVAL), (dict(c=None), bg.BERGSON_EINVAL),
    (dict(r=FAKE + 2), bg.BERGSON_EALIGN), (dict(state_kind=0, v=FAKE + 2), bg.BERGSON_EALIGN),
    (dict(ws=None), bg.BERGSON_EINVAL), (dict(ws=FAKE + 8), bg.BERGSON_EALIGN),
    (dict(ws_bytes=100), bg.BERGSON_EWORKSPACE), (dict(n_mats=-1), bg.BERGSON_EINVAL),
])
def test_moment_refusals(kw, code):
    assert moments(**kw) == code and bg.bergson_last_error() != ""


def test_moment_calls_that_pass():
    for st in (moments(), moments(state_kind=0, v_scale=None), moments(v=FAKE + 1)):
        assert accepted(st), bg.bergson_last_error()
    assert bg.lib().bergson_factor_moments_workspace(None, 1, ctypes.byref(ctypes.c_size_t())) == \
        bg.BERGSON_EINVAL


def test_binding_refuses_what_it_cannot_pass_on():
    f = torch.zeros((4, 6))
    i = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        bg.bergson_token_logprobs(f.double(), i, 1.0, f[:, 0], f[:, 0])
    with pytest.raises(ValueError):
        bg.bergson_token_logprobs(f.t(), i, 1.0, f[:, 0], f[:, 0])
    with pytest.raises(ValueError):
        bg.bergson_token_logprobs_backward(f, i, 1.0, f[0], None, f[0], None, torch.zeros((4, 5)))
    with pytest.raises(ValueError):
        bg.bergson_preference_loss(torch.zeros((3, 6)), None, None, 0, 0.1, 0.0, 0.0, False, f, f,
                                   None, torch.zeros((3, 6)))
    p = torch.zeros(300)
    with pytest.raises(ValueError):                       # one scale of two
        bg.AdamWTensor(p, p, p, p, m_scale=torch.zeros(2)).to_c()
    with pytest.raises(ValueError):                       # a scale per 256 elements
        u = torch.zeros(300, dtype=torch.uint8)
        bg.AdamWTensor(p, p, u, u, m_scale=torch.zeros(1), v_scale=torch.zeros(2)).to_c()
    with pytest.raises(ValueError):
        bg.AdamWTensor(p, p, p.half(), p).to_c()
    with pytest.raises(ValueError):                       # 32-bit indices
        bg.bergson_token_logprobs(f, i.int(), 1.0, f[:, 0].contiguous(), f[:, 0].contiguous())
    with pytest.raises(ValueError):
        bg.bergson_token_logprobs(f, i, 1.0, p[:3], p[:4])
    with pytest.raises(ValueError):                       # a mask of another shape, of another type
        bg.bergson_preference_loss(f, None, torch.ones((4, 5), dtype=torch.uint8), 0, 0.1, 0.0, 0.0,
                                   False, p[:1], p[:2], None, f)
    with pytest.raises(ValueError):
        bg.bergson_preference_loss(f, None, torch.ones((4, 6), dtype=torch.bool), 0, 0.1, 0.0, 0.0,
                                   False, p[:1], p[:2], None, f)
    with pytest.raises(ValueError):
        bg.bergson_policy_loss(f, f[:3], None, None, p[:4], None, 0.2, 0.2, 0.0, 0.0, 0, 1.0, p[:1],
                               None, None, f, None, p)
    with pytest.raises(ValueError):
        bg.bergson_policy_loss(f, f, None, None, p[:3], None, 0.2, 0.2, 0.0, 0.0, 0, 1.0, p[:1],
                               None, None, f, None, p)
    with pytest.raises(ValueError):
        bg.AdamWTensor(p, p[:10], p, p).to_c()
    with pytest.raises(ValueError):
        bg.AdamWTensor(torch.zeros(600)[::2], p, p, p).to_c()
    with pytest.raises(ValueError):
        bg.MomentMatrix(torch.zeros(4, 6), torch.zeros(5), torch.zeros(6)).to_c()
    with pytest.raises(ValueError):
        bg.MomentMatrix(torch.zeros(4, 6), torch.zeros(4), torch.zeros(6), torch.zeros(1)).to_c()


def test_workspaces_grow_with_the_work():
    a = bg.bergson_policy_loss_workspace(1, 1)
    b = bg.bergson_policy_loss_workspace(4096, 8192)
    assert 0 < a < b and math.isfinite(b) and b < 4096 * 8192
    m = [bg.bergson_moment_matrix(FAKE, None, 4096, 4096, FAKE, FAKE, 0, 0)]
    assert 0 < bg.bergson_factor_moments_workspace(m) < 4096 * 4096 * 4 // 8


class FakeTensor:
    """What the binding asks of a device tensor, without a device."""
    is_cuda = True

    def __init__(self, shape, strides, dtype=torch.float32):
        self.shape, self.strides, self.dtype = torch.Size(shape), strides, dtype

    def stride(self):
        return self.strides

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return FAKE


@pytest.mark.parametrize("T,strides", [(6, (0, 1)), (1, (0, 1)), (1, (0, 0))])
def test_advantages_that_sequences_share_are_refused(T, strides):
    """One row for all sequences has leading dimension 0, which the C call takes for [B] advantages: it
    would read past the row."""
    x, one = FakeTensor((4, T), (T, 1)), FakeTensor((1,), (1,))
    ws = FakeTensor((1 << 20,), (1,), torch.uint8)

    def call(adv):
        bg.bergson_policy_loss(x, x, None, None, adv, None, 0.2, 0.2, 0.0, 0.0, 0, 1.0, one, None,
                               None, x, None, ws, stream=0)
    with pytest.raises(ValueError, match="advantages"):
        call(FakeTensor((4, T), strides))
    for adv in (FakeTensor((4,), (1,)), x):
        with pytest.raises(bg.BergsonError):          # the injected status: past the checks
            call(adv)


def test_gradient_scales_of_other_types_are_refused():
    """They would be read as the bits of an fp32 number."""
    def call(gs):
        bg.bergson_adamw_step([], 1e-3, 0.9, 0.99, 1e-8, 1, grad_scale=gs, stream=0)
    for dtype in (torch.float64, torch.bfloat16, torch.float16, torch.int32):
        with pytest.raises(ValueError, match="grad_scale"):
            call(FakeTensor((1,), (1,), dtype))
    with pytest.raises(ValueError, match="grad_scale"):
        call(FakeTensor((2,), (1,)))
    for gs in (None, FAKE, FakeTensor((1,), (1,)), FakeTensor((), ())):
        with pytest.raises(bg.BergsonError):          # the injected status: past the checks
            call(gs)


class Host(FakeTensor):
    """... of a tensor in host memory."""
    is_cuda, device = False, "cpu"

    def __init__(self, t, pinned=False):
        super().__init__(t.shape, t.strides, t.dtype)
        self.pinned = pinned

    def is_pinned(self):
        return self.pinned


def _device_calls():
    """Every training-side call of the binding as (its tensors by name, the call of them)."""
    x, v, one, three = (FakeTensor(s, st) for s, st in (((4, 6), (6, 1)), ((4,), (1,)), ((1,), (1,)),
                                                        ((3,), (1,))))
    two = FakeTensor((2,), (1,))
    idx, mask = FakeTensor((4,), (1,), torch.int64), FakeTensor((4, 6), (6, 1), torch.uint8)
    ws = FakeTensor((1 << 20,), (1,), torch.uint8)
    u = FakeTensor((4,), (1,), torch.uint8)
    r, c = v, FakeTensor((6,), (1,))
    return {
        "logprobs": (dict(logits=x, targets=idx, logp=v, lse=v, entropy=v),
                     lambda t: bg.bergson_token_logprobs(t["logits"], t["targets"], 1.0, t["logp"],
                                                         t["lse"], t["entropy"], stream=0)),
        "backward": (dict(logits=x, targets=idx, lse=v, entropy=v, d_logp=v, d_entropy=v, d_logits=x),
                     lambda t: bg.bergson_token_logprobs_backward(
                         t["logits"], t["targets"], 1.0, t["lse"], t["entropy"], t["d_logp"],
                         t["d_entropy"], t["d_logits"], stream=0)),
        "policy": (dict(logp=x, old_logp=x, ref_logp=x, entropy=x, advantages=v, mask=mask, loss=one,
                        seq_loss=v, stats=three, d_logp=x, d_entropy=x, workspace=ws),
                   lambda t: bg.bergson_policy_loss(
                       t["logp"], t["old_logp"], t["ref_logp"], t["entropy"], t["advantages"], t["mask"],
                       0.2, 0.2, 0.1, 0.1, 0, 1.0, t["loss"], t["seq_loss"], t["stats"], t["d_logp"],
                       t["d_entropy"], t["workspace"], stream=0)),
        "preference": (dict(logp=x, ref_logp=x, mask=mask, loss=one, pair_loss=two, rewards=v, d_logp=x),
                       lambda t: bg.bergson_preference_loss(
                           t["logp"], t["ref_logp"], t["mask"], 0, 0.1, 0.0, 0.0, False, t["loss"],
                           t["pair_loss"], t["rewards"], t["d_logp"], stream=0)),
        "adamw": (dict(param=v, grad=v, m=u, v=u, master=v, m_scale=one, v_scale=one, grad_scale=one),
                  lambda t: bg.bergson_adamw_step(
                      [bg.AdamWTensor(t["param"], t["grad"], t["m"], t["v"], t["master"], t["m_scale"],
                                      t["v_scale"])], 1e-3, 0.9, 0.99, 1e-8, 1,
                      grad_scale=t["grad_scale"], stream=0)),
        "values": (dict(codes=u, scale=one, out=v),
                   lambda t: bg.bergson_adamw_state_values(t["codes"], t["scale"], 0, t["out"], stream=0)),
        "moments": (dict(v=x, r=r, c=c, workspace=ws),
                    lambda t: bg.bergson_factor_moments([bg.MomentMatrix(t["v"], t["r"], t["c"])], 1.0,
                                                        1e-12, t["workspace"], stream=0)),
    }


@pytest.mark.parametrize("name", list(_device_calls()))
def test_tensors_in_host_memory_are_refused(name):
    """A kernel would follow their addresses.  Pinned memory, which a device can read, passes."""
    tensors, call = _device_calls()[name]
    with pytest.raises(bg.BergsonError):              # the injected status: past the checks
        call(tensors)
    for what, t in tensors.items():
        with pytest.raises(ValueError, match=f"^{what} must be on a CUDA device"):
            call({**tensors, what: Host(t)})
        with pytest.raises(bg.BergsonError):
            call({**tensors, what: Host(t, pinned=True)})


@pytest.mark.parametrize("name", list(_device_calls()))
def test_device_tensors_of_other_sizes_are_refused_by_name(name):
    tensors, call = _device_calls()[name]
    first = next(iter(tensors))                       # the others' sizes follow from it
    for what, t in tensors.items():
        if what in (first, "workspace"):
            continue
        wrong = FakeTensor((t.shape[0] + 300, *t.shape[1:]), t.strides, t.dtype)
        with pytest.raises(ValueError, match=f"^{what} must be "):
            call({**tensors, what: wrong})
        with pytest.raises((ValueError, TypeError)):
            call({**tensors, what: FakeTensor(t.shape, t.strides, torch.float64)})


@pytest.mark.parametrize("kind,record", [("bergson_policy_args", "_POLICY_RECORD"),
                                         ("bergson_preference_args", "_PREFERENCE_RECORD")])
def test_packed_records_have_the_fields_places(kind, record):
    from paper_2606_11660_gb300 import binding
    kind, record = getattr(bg, kind), getattr(binding, record)
    fields = kind._fields_
    values = [k + 1.5 if t is ctypes.c_double else k + 1 for k, (_, t) in enumerate(fields)]
    assert record.size == ctypes.sizeof(kind)
    packed = kind.from_buffer_copy(record.pack(*values))
    assert [getattr(packed, name) for name, _ in fields] == values


@pytest.mark.parametrize("name,missing", [("policy", ("old_logp", "loss", "d_logp")),
                                          ("preference", ("loss", "pair_loss", "d_logp"))])
def test_missing_tensors_are_the_librarys_to_refuse(name, missing):
    tensors, call = _device_calls()[name]
    bg.bergson_debug_inject_status(0, 0)
    for what in missing:
        with pytest.raises(bg.BergsonError, match="EINVAL"):
            call({**tensors, what: None})
