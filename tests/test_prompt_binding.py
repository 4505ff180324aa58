"""The native marshalling of the prompt pass: host tensors, wrong types, shapes
and layouts raise before anything is launched."""
import pytest
import torch

from paper_2607_16673_amd import binding as B


def _calls(dev, dt=torch.bfloat16):
    z = lambda *s, dtype=dt: torch.zeros(*s, dtype=dtype, device=dev)
    f = lambda *s: torch.zeros(*s, device=dev)
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)
    pre = dict(q=z(20, 2, 64), k=z(20, 2, 64), v=z(20, 4, 32), alpha=f(20, 4) + 1, beta=f(20, 4), seq_start=i(0, 5, 20),
               out=z(20, 4, 32), state_out=f(2, 4, 64, 32), state=f(2, 4, 64, 32), workspace=None, status=i(0, 0))
    if dev != "cpu":
        pre["workspace"] = B.prefill_workspace(pre["q"], pre["v"], 2)
    conv = dict(x=z(20, 16), weight=f(16, 4), seq_start=i(0, 5, 20), y=z(20, 16), conv_state_out=f(2, 3, 16),
                conv_state=f(2, 3, 16), bias=f(16), status=i(0, 0))
    inp = dict(q=z(20, 2, 64), k=z(20, 2, 64), a=z(20, 4), b=z(20, 4), a_log=f(4), dt_bias=f(4), q_out=z(20, 4, 64),
               k_out=z(20, 4, 64), alpha=f(20, 4), beta=f(20, 4))
    norm = dict(x=f(20, 4, 32), z=z(20, 4, 32), weight=f(32), y=z(20, 4, 32))
    fns = dict(prefill=B.sla_prefill, conv=B.sla_conv_prefill, inputs=B.sla_recurrent_inputs, norm=B.sla_gated_norm)
    return {n: (lambda fn=fns[n], a=a, **o: fn(**{**a, **o}), a)
            for n, a in dict(prefill=pre, conv=conv, inputs=inp, norm=norm).items()}


NAMES = ["prefill", "conv", "inputs", "norm"]
OPTIONAL = {"status", "workspace", "state", "conv_state", "bias", "dt_bias", "weight"}
STRIDED = {"q", "k", "v", "x", "z", "a", "b"}  # (the norm's x is dense)


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_and_non_tensors_are_refused(name):
    call, tensors = _calls("cpu")[name]
    with pytest.raises(ValueError, match="must live on"):
        call()
    for key in tensors:
        with pytest.raises((TypeError, ValueError)):
            call(**{key: [1, 2]})


@pytest.mark.parametrize("name,word", [("prefill", "family"), ("norm", "gate")])
def test_unknown_words_are_refused(name, word):
    with pytest.raises(KeyError):
        _calls("cpu")[name][0](**{word: "other"})


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_wrong_types_shapes_and_layouts_are_refused(name):
    call, tensors = _calls("cuda")[name]
    call()
    for key, t in tensors.items():
        if t is None:
            continue
        bad = [t.double() if t.is_floating_point() else t.long(), t.cpu(), t.repeat_interleave(2, -1)[..., ::2], t[None, None]]
        if key not in ("workspace", "seq_start", "weight"):
            bad.append(t[:1])
        if t.dim() == 3 and key in STRIDED:
            bad.append(t.transpose(1, 2).contiguous().transpose(1, 2))
        for x in bad:
            with pytest.raises((TypeError, ValueError)):
                call(**{key: x})
        if key not in OPTIONAL:
            with pytest.raises((TypeError, ValueError, B.SlaError)):
                call(**{key: None})
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_library_refusals_name_the_call():
    calls = _calls("cuda")
    with pytest.raises(B.SlaError, match="sla_prefill"):
        calls["prefill"][0](workspace=None)
    with pytest.raises(B.SlaError, match="sla_prefill"):
        calls["prefill"][0](family="gla")
    with pytest.raises(B.SlaError, match="sla_conv_prefill"):
        calls["conv"][0](y=calls["conv"][1]["x"])
    with pytest.raises(B.SlaError, match="sla_recurrent_inputs"):
        calls["inputs"][0](eps=-1.0)
    with pytest.raises(B.SlaError, match="sla_gated_norm"):
        calls["norm"][0](eps=float("nan"))
    torch.cuda.synchronize()
