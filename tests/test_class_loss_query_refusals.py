"""The workspace query of the losses over a linear layer's classes: sizes and strides that the calls refuse, before any device is touched; and the same by way of tensors."""

import pytest

from paper_2403_11204_amd import api

P = 0x100000          # an address that is never followed


def size(x=P, ldx=64, w=P, ldw=64, dt=1, rows=10, classes=300, dim=64, top=0, outputs=7):
    return api.lib().slp_linear_loss_workspace_bytes(x, ldx, w, ldw, dt, rows, classes, dim, top, outputs)


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("name", ["ldx", "ldw"])
def test_strides(name, dt):
    assert size(dt=dt) > 0
    for ld in (0, 1, 63, -1, -64, -(1 << 40), (1 << 20) + 8, 5000000, 1 << 23, 1 << 40, (1 << 62)):
        assert size(dt=dt, **{name: ld}) == 0, ld
    assert size(dt=dt, **{name: 1 << 20}) > 0
    # a single row may have any stride up to the largest of all
    single = dict(rows=1) if name == "ldx" else dict(classes=1)
    assert size(dt=dt, **single, **{name: 1 << 40}) > 0 and size(dt=dt, **single, **{name: 0}) == 0 and size(dt=dt, **single, **{name: (1 << 40) + 8}) == 0


def test_sizes():
    for bad in (dict(rows=-1), dict(rows=0), dict(classes=0), dict(dim=0), dict(dt=2), dict(top=-1), dict(top=1025), dict(rows=(1 << 20) + 1), dict(classes=(1 << 24) + 1), dict(dim=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21),
                dict(rows=1 << 20, classes=1 << 20), dict(classes=1 << 14, dim=1 << 20, ldx=1 << 20, ldw=1 << 20), dict(rows=1 << 16, top=1024), dict(rows=1 << 14, dim=1 << 20, ldx=1 << 20, ldw=1 << 20),
                dict(rows=1 << 20, dim=2048, ldx=2048, ldw=2048), dict(x=P + 1), dict(w=P + 1)):
        assert size(**bad) == 0, bad
    assert size(rows=1 << 20, dim=2048, ldx=2048, ldw=2048, outputs=1) > 0            # (rows of 4 GiB: dw alone is refused)


def test_the_calls_refuse_the_same():
    """Whatever the query answers with 0, the call answers with an error, in front of any work."""
    for bad in (dict(ldw=0), dict(ldw=5000000), dict(ldx=0), dict(ldw=-64), dict(rows=1 << 20, classes=1 << 20), dict(x=P + 1)):
        assert size(**bad) == 0
        a = dict(x=P, ldx=64, w=P, ldw=64, bias=None, dt=1, rows=10, classes=300, dim=64, y=P, id_bytes=4, scale=1.0, loss=P, losses=P, lse=P, dx=P, lddx=64, dw=P, lddw=64, dw_dt=0, dbias=None, work=None, size=0)
        a.update(bad)
        assert api.lib().slp_linear_cross_entropy(*a.values(), None) < 0


@pytest.mark.gpu
def test_tensors_with_such_strides():
    import torch
    x, y = torch.ones(10, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(10, dtype=torch.int32, device="cuda")
    w = torch.ones(300, 64, dtype=torch.bfloat16, device="cuda")
    top, ids = torch.zeros(10, 3, device="cuda"), torch.zeros(10, 3, dtype=torch.int32, device="cuda")
    wide = torch.ones(2, (1 << 20) + 8, dtype=torch.bfloat16, device="cuda")[:, :64]
    for bad in ((x, w[:1].expand(300, 64)), (x[:1].expand(10, 64), w), (x, wide)):
        with pytest.raises(api.SlpError):
            api.linear_cross_entropy(*bad, y)
        with pytest.raises(api.SlpError):
            api.linear_distillation(*bad, top, ids)
    r = api.linear_cross_entropy(x, w, y)
    assert ((r.losses - 5.703782474656201).abs() < 1e-5).all()        # (300 equal logits)
