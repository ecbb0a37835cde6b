"""AdamW and the losses on a host without a GPU: sizes, and refusals that come before any CUDA call."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def meq():
    from paper_2609_35701_gb300 import build

    build.build()
    from paper_2609_35701_gb300 import meq as m

    return m


def test_adamw_state_bytes(meq):
    shapes = [(1, 1), (1, 256), (3, 171)]                      # 256, 256 and 768 padded elements
    p32, w32 = meq.adamw_state_bytes(shapes)
    p8, w8 = meq.adamw_state_bytes(shapes, state_bits=8)
    assert p32 == 8 * 1280 and p8 == 2 * 1280 + 2 * 4 * 5 and w32 > 0 and w8 > 0
    # a quarter of the moments of a 130M model, and 1/64 more for the scales
    big = [(32000, 768)] * 2 + [(768, 768)] * 48 + [(2048, 768)] * 36
    p32, _ = meq.adamw_state_bytes(big)
    p8, _ = meq.adamw_state_bytes(big, state_bits=8, param_dtype="bfloat16", grad_dtype="bfloat16")
    assert p8 * 4 == p32 + p32 // 64


def test_adamw_refusals(meq):
    for kw in (dict(state_bits=4), dict(beta1=-0.1), dict(beta2=1.0), dict(eps=0.0), dict(eps=1e-40), dict(beta1=float("nan"))):
        with pytest.raises(meq.MeqError) as e:
            meq.adamw_state_bytes([(4, 4)], **kw)
        assert e.value.status == 1
    for bad in ([], [(0, 4)], [(1, (1 << 20) + 1)]):
        with pytest.raises(meq.MeqError) as e:
            meq.adamw_state_bytes(bad)
        assert e.value.status == 1
    with pytest.raises(ValueError):
        meq.adamw_state_bytes([(4, 4)], param_dtype="float64")
    with pytest.raises(KeyError):
        meq.adamw_state_bytes([(4, 4)], momentum=0.9)
    st = ctypes.c_void_p()
    decay = (ctypes.c_float * 1)(-1.0)
    assert meq.lib.meq_adamw_init(meq._shape_array([(4, 4)]), decay, 1, None, None, ctypes.byref(st)) == 1 and not st.value
    assert b"decay" in meq.lib.meq_adamw_last_error(None)
    assert meq.lib.meq_adamw_init(meq._shape_array([(4, 4)]), None, 1, None, None, None) == 1
    for call in (lambda: meq.lib.meq_adamw_step(None, None, None, None, 0.1, 0.0, None, None),
                 lambda: meq.lib.meq_adamw_grad_norm(None, None, 1.0, None, None), lambda: meq.lib.meq_adamw_sync(None),
                 lambda: meq.lib.meq_adamw_read_values(None, None, None, None), lambda: meq.lib.meq_adamw_set_steps(None, 0)):
        assert call() == 1
        assert b"state is NULL" in meq.lib.meq_adamw_last_error(None)
    assert meq.lib.meq_adamw_free(None) == 0


FAKE = 4096  # never dereferenced: the checks are host-only
F32, BF16 = 0, 1


def test_logits_refusals(meq):
    fn = meq.lib.meq_token_logprobs
    cases = [
        ((FAKE, 7, 4, 4, 4, FAKE, FAKE, FAKE), b"meq_dtype"),
        ((FAKE, F32, -1, 4, 4, FAKE, FAKE, FAKE), b"rows"),
        ((FAKE, F32, (1 << 27) + 1, 4, 4, FAKE, FAKE, FAKE), b"rows"),
        ((FAKE, F32, 4, 0, 4, FAKE, FAKE, FAKE), b"cols"),
        ((FAKE, F32, 4, (1 << 28) + 1, 1 << 29, FAKE, FAKE, FAKE), b"cols"),
        ((FAKE, F32, 4, 4, 3, FAKE, FAKE, FAKE), b"stride"),
        ((None, F32, 4, 4, 4, FAKE, FAKE, FAKE), b"NULL"),
        ((FAKE, F32, 4, 4, 4, None, FAKE, FAKE), b"NULL"),
        ((FAKE, F32, 4, 4, 4, FAKE, None, FAKE), b"NULL"),
        ((FAKE + 2, F32, 4, 4, 4, FAKE, FAKE, FAKE), b"aligned"),
        ((FAKE + 1, BF16, 4, 4, 4, FAKE, FAKE, FAKE), b"aligned"),
        ((FAKE, F32, 4, 4, 4, FAKE + 4, FAKE, FAKE), b"aligned"),
        ((FAKE, F32, 4, 4, 4, FAKE, FAKE, FAKE + 1), b"aligned"),
    ]
    for args, text in cases:
        assert fn(*args, None) == 1, args
        assert text in meq.lib.meq_last_error(None), (args, meq.lib.meq_last_error(None))
    assert fn(None, F32, 0, 4, 4, None, None, None, None) == 0  # no rows: nothing to do


def test_loss_refusals(meq):
    def policy(**kw):
        a = dict(logits=FAKE, type=F32, rows=4, cols=4, ld=4, targets=FAKE, old=FAKE, adv=FAKE, w=None, ref=FAKE, lo=0.2, hi=0.2, kl=0.1,
                 sums=FAKE, logp=FAKE, grad=FAKE, ldg=4, scale=None, work=FAKE, stream=None)
        a.update(kw)
        return meq.lib.meq_policy_loss(*a.values())

    for kw, text in ((dict(old=None), b"old_logp"), (dict(adv=None), b"advantages"), (dict(ref=None), b"ref_logp"), (dict(sums=None), b"sums"),
                     (dict(work=None), b"work"), (dict(work=FAKE + 8), b"work"), (dict(ldg=3), b"stride"), (dict(lo=-0.1), b"clip_low"),
                     (dict(lo=1.1), b"clip_low"), (dict(hi=float("nan")), b"clip_high"), (dict(kl=-1.0), b"kl_coef"),
                     (dict(grad=FAKE + 2), b"aligned"), (dict(scale=FAKE + 1), b"aligned"), (dict(w=FAKE + 2), b"aligned")):
        assert policy(**kw) == 1 and text in meq.lib.meq_last_error(None), (kw, meq.lib.meq_last_error(None))

    def preference(**kw):
        a = dict(logits=FAKE, type=F32, rows=4, cols=4, ld=4, targets=FAKE, starts=FAKE, pairs=1, ref=FAKE, w=None, beta=0.1, smooth=0.0,
                 loss=FAKE, margins=FAKE, logp=FAKE, grad=FAKE, ldg=4, scale=None, work=FAKE, stream=None)
        a.update(kw)
        return meq.lib.meq_preference_loss(*a.values())

    for kw, text in ((dict(pairs=0), b"pairs"), (dict(starts=None), b"starts"), (dict(ref=None), b"ref_logp"), (dict(loss=None), b"loss"),
                     (dict(margins=None), b"margins"), (dict(beta=0.0), b"beta"), (dict(beta=float("inf")), b"beta"),
                     (dict(smooth=1.5), b"label_smoothing"), (dict(starts=FAKE + 4), b"aligned"), (dict(work=None), b"work")):
        assert preference(**kw) == 1 and text in meq.lib.meq_last_error(None), (kw, meq.lib.meq_last_error(None))
    assert meq.lib.meq_loss_work_floats(10, 3) >= 7 * 10 + 3 and meq.lib.meq_loss_work_floats(-1, 0) == 0


def test_binding_refuses_host_tensors(meq):
    z, t, v = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for call in (lambda: meq.token_logprobs(z, t), lambda: meq.policy_loss(z, t, v, v), lambda: meq.preference_loss(z, t, t, v)):
        with pytest.raises(ValueError):
            call()
