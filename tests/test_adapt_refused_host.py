"""Adapters that the entry point would refuse are refused where they are given, ahead of a prefix that is encoded with them."""
import pytest
import torch

from test_sampled_drafting import host_drafter  # noqa: F401 (a fixture)

BF16 = torch.bfloat16


def test_types_places_and_layouts(host_drafter):  # noqa: F811
    d = host_drafter
    a, b, s = torch.zeros(3, 16, 64, dtype=BF16), torch.zeros(3, 1000, 16, dtype=BF16), torch.ones(3)
    off = torch.zeros(3 * 16 * 64 + 4, dtype=BF16)[4:].view(3, 16, 64)               # (contiguous, but 8 bytes from an aligned address)
    assert a.data_ptr() % 16 == 0 and off.data_ptr() % 16 == 8
    d.adapt(a, b, s, which=1)
    kept = d._adapters
    for bad in (dict(scale=s.double()), dict(scale=s.to(BF16)), dict(scale=torch.ones(6)[::2]), dict(scale=s.to("meta")), dict(scale=torch.ones(4)[1:]),
                dict(lora_a=torch.zeros(3, 64, 16, dtype=BF16).transpose(1, 2)), dict(lora_b=torch.zeros(3, 16, 1000, dtype=BF16).transpose(1, 2)),
                dict(lora_a=a.to("meta")), dict(lora_b=b.to("meta")), dict(lora_a=off)):
        with pytest.raises(ValueError):
            d.adapt(**{**dict(lora_a=a, lora_b=b, scale=s), **bad})
        assert d._adapters is kept
