"""CPU-only checks of the operators for language models: what their entry points refuse, on the host and before any GPU work."""
import math

import numpy as np
import pytest

from paper_2311_06281_amd import binding as hb

P = 4096  # a non-null, aligned fake address: a refused call never touches it
INVALID, UNSUPPORTED = hb.HEINSEN_ERR_INVALID_ARG, hb.HEINSEN_ERR_UNSUPPORTED


def refused(status, call, *args, **more):
    with pytest.raises(hb.HeinsenError) as e:
        call(*args, **more)
    assert e.value.status == status


ATTENTION = dict(q=P, k=P, v=P, log_a=P, s0=P, out=P, sn=P, B=1, n=8, H=4, K=16, V=16, scale=1.0, flags=0)
BACKWARD = {m: x for m, x in ATTENTION.items() if m not in ("out", "sn")} | dict(
    grad_out=P, grad_sn=P, grad_q=P, grad_k=P, grad_v=P, grad_log_a=P, grad_s0=P)

BAD_ATTENTION = [
    (dict(q=0), INVALID), (dict(k=None), INVALID), (dict(v=0), INVALID),
    (dict(B=0), INVALID), (dict(n=0), INVALID), (dict(H=0), INVALID), (dict(K=0), INVALID), (dict(V=-1), INVALID), (dict(Hk=0), INVALID),
    (dict(Hk=3), INVALID),                                                 # 4 heads of v over 3 of q
    (dict(K=129), UNSUPPORTED), (dict(V=200), UNSUPPORTED),
    (dict(flags=hb.HEINSEN_POSITIVE), INVALID), (dict(flags=hb.HEINSEN_GATE_SIGMOID), INVALID), (dict(flags=1 << 20), INVALID),
    (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(q=P + 2), INVALID), (dict(k=P + 1, flags=hb.HEINSEN_IN_BF16), INVALID), (dict(log_a=P + 2), INVALID), (dict(s0=P + 2), INVALID),
    (dict(starts=P + 4), INVALID),
    (dict(q_stride=63), INVALID), (dict(k_stride=-64), INVALID), (dict(v_stride=1), INVALID), (dict(v_stride=1 << 40), UNSUPPORTED),
    (dict(B=1 << 30), UNSUPPORTED), (dict(H=1 << 40, Hk=1), UNSUPPORTED), (dict(n=1 << 40), UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", BAD_ATTENTION + [(dict(out=0), INVALID), (dict(out=P + 2), INVALID), (dict(sn=P + 1), INVALID)])
def test_attention_refuses(change, status):
    refused(status, hb.heinsen_linear_attention, **(ATTENTION | change))


@pytest.mark.parametrize("change,status", BAD_ATTENTION + [
    (dict(grad_out=0), INVALID), (dict(grad_q=0), INVALID), (dict(grad_k=None), INVALID), (dict(grad_v=0), INVALID),
    (dict(log_a=None), INVALID),                                           # a gradient of what there is not
    (dict(grad_out=P + 2), INVALID), (dict(grad_sn=P + 2), INVALID), (dict(grad_s0=P + 2), INVALID), (dict(grad_log_a=P + 2), INVALID),
])
def test_attention_backward_refuses(change, status):
    refused(status, hb.heinsen_linear_attention_backward, **(BACKWARD | change))


NORM = dict(u=P, gate=P, residual=P, scale=P, w_post=P, w_pre=P, h=P, y=P, rows=4, D=64, eps=1e-6, flags=0)
NORM_BACKWARD = {m: x for m, x in NORM.items() if m not in ("h", "y")} | dict(
    grad_h=P, grad_y=P, grad_u=P, grad_gate=P, grad_residual=P, grad_scale=P, grad_w_post=P, grad_w_pre=P)

BAD_NORM = [
    (dict(u=0), INVALID), (dict(rows=0), INVALID), (dict(D=0), INVALID), (dict(D=16385), UNSUPPORTED), (dict(rows=1 << 50), UNSUPPORTED),
    (dict(w_pre=None), INVALID),
    (dict(flags=hb.HEINSEN_DECAY_PER_HEAD), INVALID), (dict(flags=1 << 20), INVALID),
    (dict(eps=-1e-6), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID),
    (dict(u=P + 2), INVALID), (dict(gate=P + 1, flags=hb.HEINSEN_IN_BF16), INVALID), (dict(residual=P + 2), INVALID),
    (dict(scale=P + 2), INVALID), (dict(w_post=P + 2), INVALID),
    (dict(u_stride=63), INVALID), (dict(gate_stride=-1), INVALID), (dict(u_stride=1 << 30), UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", BAD_NORM + [(dict(h=None, y=None), INVALID), (dict(h=P + 2), INVALID), (dict(y=P + 2), INVALID)])
def test_block_norm_refuses(change, status):
    refused(status, hb.heinsen_block_norm, **(NORM | change))


@pytest.mark.parametrize("change,status", BAD_NORM + [
    (dict(grad_h=None, grad_y=None), INVALID), (dict(grad_u=None), INVALID), (dict(gate=None), INVALID), (dict(residual=None), INVALID),
    (dict(scale=None), INVALID), (dict(w_post=None), INVALID), (dict(grad_y=None, w_pre=None), INVALID),
    (dict(grad_h=P + 2), INVALID), (dict(grad_u=P + 2), INVALID), (dict(grad_w_pre=P + 2), INVALID),
])
def test_block_norm_backward_refuses(change, status):
    refused(status, hb.heinsen_block_norm_backward, **(NORM_BACKWARD | change))


# a token's gradients of its own heads' q and k, which are added up afterwards, have to lie within 32 bits for a chunk of tokens
def test_attention_backward_refuses_too_many_shared_heads():
    shared = BACKWARD | dict(H=1 << 17, Hk=1 << 10, K=128, V=1)
    refused(UNSUPPORTED, hb.heinsen_linear_attention_backward, **shared)


def test_the_scan_refuses_the_operators_flags():
    for flag in (hb.HEINSEN_DECAY_PER_HEAD, hb.HEINSEN_GATE_SIGMOID):
        assert hb.heinsen_scan_status(P, P, P, P, 1, 1, 8, 0, flag) == INVALID


class _Tensor:
    def __init__(self, at):
        self.at = at

    def data_ptr(self):
        return self.at


class _Stream:
    cuda_stream = 0


# tensors or addresses, numbers or what converts to them: one argument that is refused shows that each arrives in its place
@pytest.mark.parametrize("direct", [True, False])
@pytest.mark.parametrize("call,arguments,bad", [(hb.heinsen_linear_attention, ATTENTION, BAD_ATTENTION), (hb.heinsen_linear_attention_backward, BACKWARD, BAD_ATTENTION),
                                                (hb.heinsen_block_norm, NORM, BAD_NORM), (hb.heinsen_block_norm_backward, NORM_BACKWARD, BAD_NORM)])
def test_arguments_of_every_kind(monkeypatch, call, arguments, bad, direct):
    hb.load()
    if not direct:
        monkeypatch.setattr(hb, "_call", hb._Converted)
    counts = {"B", "n", "H", "K", "V", "Hk", "rows", "D", "flags"} | {m + "_stride" for m in ("q", "k", "v", "u", "gate")}
    plain = {"scale", "eps", "starts"} if "K" in arguments else {"eps"}
    for change, status in bad:
        whole = arguments | change
        tensors = {m: x if m in counts | plain or x is None else _Tensor(x) for m, x in whole.items()}
        refused(status, call, **tensors, stream=_Stream())
        refused(status, call, **{m: np.int64(x) if m in counts else x for m, x in whole.items()}, stream=0)
    with pytest.raises(TypeError):
        call(**(arguments | {"q" if "q" in arguments else "u": object()}))
