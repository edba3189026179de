"""Which written views are taken: those whose elements do not overlap, every second row or
channel of a tensor among them.  No GPU: a call with a bad epsilon is refused after its
views, so the code says whether they passed."""
import pytest
import torch

import paper_1903_06681_amd as dc

A, B = 0x10000, 0x20000


def verdict(t):
    n, c, h, w = t.shape
    good = dc.View(n, c, h, w, c * h * w, h * w, w, dc.DC_F32)
    with pytest.raises(dc.DcError) as e:
        dc.norm_fwd(good, A, None, None, -1.0, dc.View.of(t), B, None, None, 0)
    return {-10: "taken", -2: "overlap"}[e.value.status]


T = torch.empty(3, 5, 7, 9)


@pytest.mark.parametrize("name", ["rows", "rows_columns", "channels", "samples", "all", "last_plane_short", "transposed"])
def test_slices_with_steps_are_taken(name):
    t = {"rows": T[:, :, ::2], "rows_columns": T[:, :, ::3, 2:4], "channels": T[:, ::2, :, :], "samples": T[::2, 1::2, 1::4],
         "all": T[::2, ::4, ::6, :1], "transposed": T.permute(1, 0, 2, 3)[:, ::2],
         # planes that start where the last row of the plane before ends
         "last_plane_short": torch.as_strided(T, (2, 2, 3, 4), (44, 22, 9, 1))}[name]
    assert verdict(t) == "taken"


@pytest.mark.parametrize("shape,strides", [((2, 2, 3, 4), (44, 21, 9, 1)), ((2, 2, 3, 4), (43, 22, 9, 1)), ((2, 2, 3, 4), (44, 22, 3, 1)),
                                           ((2, 1, 3, 4), (0, 22, 9, 1)), ((1, 2, 3, 4), (44, 9, 9, 1))])
def test_one_element_less_overlaps(shape, strides):
    assert verdict(torch.as_strided(T, shape, strides)) == "overlap"
