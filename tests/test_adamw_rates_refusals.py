"""moe_adamw refuses rates that are not five 4-byte words: the kernel reads them as four floats and an integer."""
import pytest
import torch

from paper_1701_06538_b200 import binding as B


class Reached(Exception):
    pass


@pytest.fixture
def call(monkeypatch):
    """moe_adamw with an empty list, up to where the library would be called."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)  # what a tensor of the host says of its device

    def reached():
        raise Reached

    monkeypatch.setattr(B, "lib", reached)
    return lambda rates: B.moe_adamw(B.moe_adamw_list([]), 1e-3, 0.9, 0.999, 1e-8, 1, rates=rates)


@pytest.mark.parametrize("rates", [torch.zeros(4), torch.zeros(0), torch.zeros(5, dtype=torch.float64), torch.zeros(5, dtype=torch.bfloat16), torch.zeros(20, dtype=torch.uint8),
                                   torch.zeros(5, dtype=torch.int64), torch.zeros(3, dtype=torch.float64), torch.zeros(10)[::2], torch.zeros(5, dtype=torch.bool)])
def test_refused(call, rates):
    with pytest.raises(ValueError):
        call(rates)


@pytest.mark.parametrize("rates", [None, torch.zeros(5), torch.zeros(8), torch.zeros(5, dtype=torch.int32), torch.zeros(5, dtype=torch.uint32)])
def test_taken(call, rates):
    with pytest.raises(Reached):
        call(rates)
