"""GatedUnit.check(): an expired wait is reported once; calls that went well afterwards are not blamed for it."""
import pytest

from recording_library import install, on_device


def _reported_once(unit):
    import paper_1711_09846_b200 as pbt
    unit.check()
    unit._status[4], unit._status[5] = 5, 41           # what a kernel leaves whose wait ran out
    with pytest.raises(pbt.PbtError) as e:
        unit.check()
    assert e.value.code == 5
    unit.check()
    assert not unit._status.any()


def test_an_expired_wait_is_reported_once(monkeypatch):
    import torch
    import paper_1711_09846_b200 as pbt
    install(monkeypatch)
    _reported_once(pbt.GatedUnit(on_device(torch.zeros(2, 16, 16))))


@pytest.mark.gpu
def test_an_expired_wait_is_reported_once_on_the_device():
    import torch
    import paper_1711_09846_b200 as pbt
    unit = pbt.GatedUnit(torch.randn(2, 64, 64, device="cuda", dtype=torch.bfloat16))
    with torch.cuda.stream(torch.cuda.Stream()):
        _reported_once(unit)
    unit.forward(torch.randn(2, 3, 64, device="cuda", dtype=torch.bfloat16))
    unit.check()
