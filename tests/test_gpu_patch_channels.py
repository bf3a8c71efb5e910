"""Patch rows go by the channels that the pictures have: records of gray and colour pictures have no layout, and means for other channels are refused."""
import pytest
import torch

import paper_1911_00472_amd as pkg
import pcrgen

pytestmark = pytest.mark.gpu
MEAN, ISTD = (0.485, 0.456, 0.406), (1 / 0.229, 1 / 0.224, 1 / 0.225)


def test_a_record_of_gray_and_colour_pictures_has_no_layout():
    gray = [pcrgen.make_jpeg(i, 0, 40, 24, 1, 8.0, 1, 1, 90) for i in range(2)]
    colour = [pcrgen.make_jpeg(50 + i, 1, 33, 47, 3, 6.0, 2, 2, 90) for i in range(2)]
    for files in ([gray[0], colour[0], gray[1], colour[1]], [colour[0], colour[1], gray[0]]):
        with pkg.pcr_open(pcrgen.write_record(files), 0) as r:
            with pytest.raises(pkg.PcrError) as e:
                r.patch_layout(8)
            assert e.value.code == pkg.E_UNSUPPORTED


def test_means_for_other_channels_are_refused(gray64, rgb_small):
    for data, right, wrong in ((gray64[0], 1, 3), (rgb_small[0], 3, 1)):
        with pkg.pcr_open(data, 0) as r:
            layout, pixels = r.patch_layout(8), r.decode_batch(1)
            assert pkg.patch_rows(pixels, *layout, 8, MEAN[:right], ISTD[:right])[0].shape == (layout[-1], right * 64)
            with pytest.raises(ValueError):
                pkg.patch_rows(pixels, *layout, 8, MEAN[:wrong], ISTD[:wrong])
    pixels = torch.zeros(1200, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        pkg.patch_rows(pixels, *pkg.patch_layout([(20, 20)], 3, 10), 10, MEAN[:1], ISTD[:1])
    shapes, offsets, first, rows = pkg.patch_layout([(20, 20)], 3, 10)
    assert pkg.patch_rows(pixels, shapes.clone(), offsets, first, rows, 10, MEAN, ISTD)[0].shape == (4, 300)      # tensors that come from elsewhere
