"""Layouts of handles whose record changes: a wrapper kept across a loader slot's next upload, and a handle that holds no record."""
import numpy as np
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu
MEAN, ISTD = (0.485, 0.456, 0.406), (1 / 0.229, 1 / 0.224, 1 / 0.225)


def same(a, b):
    return a[3] == b[3] and all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


def test_a_wrapper_that_is_kept_across_the_next_upload(gray64, rgb_small):
    records = [rgb_small[0], gray64[0], rgb_small[0]]
    wanted = []
    for data in records:
        with pkg.pcr_open(data, 0) as r:
            wanted.append(r.patch_layout(8, 2))
    with pkg.Loader(slots=1, slot_bytes=max(map(len, records))) as ld:
        kept = None
        for data, want in zip(records, wanted):
            ld.staging(0)[:len(data)] = np.frombuffer(data, np.uint8)
            now = ld.upload(0, len(data))
            assert kept is None or same(kept.patch_layout(8, 2), want)
            assert same(now.patch_layout(8, 2), want)
            kept = kept or now
            ld.wait(0)


def test_a_handle_without_a_record(rgb_small):
    good = torch.frombuffer(bytearray(rgb_small[0]), dtype=torch.uint8).cuda()
    bad = torch.zeros_like(good)
    with pkg.pcr_open_device(good) as r:
        with pytest.raises(pkg.PcrError):
            r.rebind_device(bad)
        shapes, offsets, first, rows = r.patch_layout(8)
        assert shapes.shape == (0, 2) and offsets.tolist() == [0] and first.tolist() == [0] and rows == 0
        for mean, istd in ((MEAN, ISTD), (MEAN[:1], ISTD[:1])):
            out, positions = pkg.patch_rows(torch.empty(0, dtype=torch.uint8, device="cuda"), shapes, offsets, first, rows, 8, mean, istd)
            assert out.shape == (0, len(mean) * 64) and positions.shape == (3, 0)
