"""Counts that are no whole numbers are refused where a Rotary is made, not cut."""
import numpy as np
import pytest
import torch

import paper_2505_17694_amd as C


@pytest.mark.parametrize("kw", [dict(axes=[16.9, 24, 24]), dict(axes=[16.0, 24, 24]), dict(axes=np.array([16.0, 24.0, 24.0])), dict(axes=["16", 24, 24]),
                                dict(axes=torch.tensor([16.5, 24.0, 24.0])), dict(axes=[None, 64]), dict(axes=64), dict(axes=[16, 16], blocks=2.0),
                                dict(blocks=2.5), dict(blocks=1.0, restart=True), dict(blocks="2"), dict(blocks=None)])
def test_fractions_are_refused(kw):
    with pytest.raises(ValueError):
        C.Rotary(128, device="cpu", **kw)


@pytest.mark.parametrize("axes", [(16, 24, 24), [16, 24, 24], np.array([16, 24, 24]), np.array([16, 24, 24], np.uint8), torch.tensor([16, 24, 24])])
def test_whole_numbers_of_any_type_pass(axes):
    rot, want = C.Rotary(128, device="cpu", axes=axes, blocks=np.int64(1)), C.Rotary(128, device="cpu", axes=[16, 24, 24])
    assert torch.equal(rot.turns, want.turns) and torch.equal(rot._axes, want._axes) and rot._fields[0][5:7] == (128, 3)
