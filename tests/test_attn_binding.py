"""The native marshalling of the attention calls: host tensors, wrong types,
shapes and layouts raise before anything is launched."""
import pytest
import torch

from paper_2607_16673_amd import binding as B


def _calls(dev, dt=torch.bfloat16):
    z = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype, device=dev)
    q, k, v = z(2, 4, 8, 64, dtype=dt), z(2, 4, 2, 64, dtype=dt), z(2, 4, 2, 64, dtype=dt)
    kc, vc = z(24, 2, 16, 64, dtype=dt), z(24, 2, 16, 64, dtype=dt)
    par = torch.arange(-1, 3, dtype=torch.int32, device=dev).repeat(2, 1)
    tab = torch.arange(24, dtype=torch.int32, device=dev).view(2, 12)  # 192 rows: more than a tile, so there is a workspace
    lens, f = z(2), z(64, dtype=torch.float32)
    ap = dict(q=q, k=k, v=v, parent_idx=par, page_table=tab, cache_len=lens, q_out=torch.empty_like(q), k_cache=kc,
              v_cache=vc, q_norm=f, k_norm=f.clone(), rope=z(50, 32, dtype=torch.float32), status=z(2))
    ve = dict(q=q, k_cache=kc, v_cache=vc, parent_idx=par, page_table=tab, cache_len=lens, out=torch.empty_like(q),
              workspace=None, status=z(2))
    co = dict(k_cache=kc, v_cache=vc, parent_idx=par, path=(par + 1).contiguous(), length=z(2) + 2, page_table=tab,
              cache_len=lens, new_len=z(2), status=z(2))
    cp = dict(k_cache=kc, v_cache=vc, src=z(2), dst=z(2) + torch.arange(1, 3, dtype=torch.int32, device=dev), rows=z(2) + 3,
              status=z(2))
    fns = dict(append=B.sla_attn_append, verify=B.sla_attn_verify, commit=B.sla_attn_commit, copy=B.sla_page_copy)
    if dev != "cpu":
        ve["workspace"] = B.attn_workspace(q, kc, tab)
    return {n: (lambda fn=fns[n], a=a, **o: fn(**{**a, **o}), a)
            for n, a in dict(append=ap, verify=ve, commit=co, copy=cp).items()}


NAMES = ["append", "verify", "commit", "copy"]
OPTIONAL = {"q_norm", "k_norm", "rope", "status", "workspace", "new_len", "rows"}


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_and_non_tensors_are_refused(name):
    call, tensors = _calls("cpu")[name]
    with pytest.raises(ValueError, match="must live on the GPU"):
        call()
    for key in tensors:
        with pytest.raises((TypeError, ValueError)):
            call(**{key: [1, 2]})


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_wrong_types_shapes_and_layouts_are_refused(name):
    call, tensors = _calls("cuda")[name]
    call()
    for key, t in tensors.items():
        if t is None:
            continue
        # a table of another width, a workspace of another size and a cache of other pages are tables, workspaces and caches
        bad = [t.double() if t.is_floating_point() else t.long(), t.cpu(), t.repeat_interleave(2, -1)[..., ::2], t[None, None]]
        if key not in ("k_cache", "v_cache", "page_table", "workspace", "rope"):
            bad.append(t[:1])
        for x in bad:
            with pytest.raises((TypeError, ValueError)):
                call(**{key: x})
        if key not in OPTIONAL:
            with pytest.raises((TypeError, ValueError, AttributeError)):
                call(**{key: None})
    with pytest.raises((TypeError, ValueError)):
        call(v_cache=tensors["v_cache"][:3])
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_other_refusals():
    calls = _calls("cuda")
    append, a = calls["append"]
    with pytest.raises(KeyError):
        append(layout="spiral")
    with pytest.raises(KeyError):
        append(topology="ring")
    with pytest.raises(ValueError):
        append(rope=torch.zeros(50, 80, device="cuda"))
    assert pytest.raises(B.SlaError, append, rope=torch.zeros(50, 24, device="cuda")).value.code == B.SLA_ERR_SHAPE
    wide = torch.zeros(2, 4, 9, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="nodes a constant step apart"):
        append(k=wide[:, :, 1:5:2])
    with pytest.raises(ValueError, match="nodes a constant step apart"):
        append(k=a["k"][:1].expand(2, -1, -1, -1))
    assert pytest.raises(B.SlaError, append, q_out=a["q"]).value.code == B.SLA_ERR_ALIAS
    verify, a = calls["verify"]
    assert pytest.raises(B.SlaError, verify, out=a["q"]).value.code == B.SLA_ERR_ALIAS
    assert pytest.raises(B.SlaError, verify, workspace=None).value.code == B.SLA_ERR_NULL
    assert pytest.raises(B.SlaError, verify, workspace=a["workspace"][:16]).value.code == B.SLA_ERR_SHAPE
    assert pytest.raises(B.SlaError, verify, scale=float("nan")).value.code == B.SLA_ERR_SHAPE
    for bad in (-1, 1 << 40):
        with pytest.raises((ValueError, B.SlaError)):
            verify(max_len=bad)
    commit, a = calls["commit"]
    assert pytest.raises(B.SlaError, commit, new_len=a["cache_len"]).value.code == B.SLA_ERR_ALIAS
    copy, a = calls["copy"]
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert pytest.raises(B.SlaError, copy, src=empty, dst=empty, rows=None, status=None).value.code in (
        B.SLA_ERR_SHAPE, B.SLA_ERR_NULL)
    torch.cuda.synchronize()
