"""Patch rows of ragged pictures against the definition in 64 bits, picture by picture.

Tolerance: the kernel computes pixel * fl(inv_std / 255) + fl(-mean * inv_std) with one multiply-add in 32 bits; the two constants are off by
2^-24 of themselves, the result by 2^-24 of itself, and pixel * inv_std / 255 <= inv_std, so before the rounding to the output's type the
error is below 2^-24 (2 inv_std + 2 |mean inv_std|) <= 2^-22 max(inv_std) (the means are below 1).  The rounding adds half a unit in the last place."""
import numpy as np
import pytest
import torch

import paper_1911_00472_amd as pkg

pytestmark = pytest.mark.gpu
MEAN, ISTD = (0.485, 0.456, 0.406), (1 / 0.229, 1 / 0.224, 1 / 0.225)
HALF_UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
SIZES = [(33, 21), (64, 64), (1, 1), (17, 130), (8, 200), (14, 14), (15, 29), (300, 7)]


def reference(pixels, sizes, C, P, m, frames):
    """float64 [rows, C * P * P], int32 [3, rows]"""
    values, places, begin = [], [], 0
    for i, (h, w) in enumerate(sizes):
        x = pixels[begin:begin + h * w * C].reshape(h, w, C).astype(np.float64)
        begin += h * w * C
        x = (x / 255 - np.array(MEAN[:C])) * np.array(ISTD[:C])
        for by in range(-(-h // (P * m))):
            for bx in range(-(-w // (P * m))):
                for iy in range(m):
                    for ix in range(m):
                        row, column = by * m + iy, bx * m + ix
                        cell = np.zeros((C, P, P))
                        part = x[row * P:(row + 1) * P, column * P:(column + 1) * P]
                        if part.size:
                            cell[:, :part.shape[0], :part.shape[1]] = part.transpose(2, 0, 1)
                        values.append(cell.reshape(-1))
                        places.append((i % frames, row, column))
    return np.array(values), np.array(places, np.int32).T


def check(got, positions, want, places):
    assert np.array_equal(positions.cpu().numpy(), places)
    tol = HALF_UNIT[got.dtype] * np.abs(want) + TINY[got.dtype] + 2.0 ** -22 * max(ISTD)
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= tol).all(), float((off - tol).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("C,P,m,frames", [(3, 14, 1, 1), (3, 16, 2, 4), (1, 8, 1, 3), (3, 7, 3, 1), (1, 5, 2, 2), (3, 1, 1, 1), (3, 28, 1, 1), (3, 128, 1, 1), (1, 16, 16, 1), (3, 100, 1, 1), (3, 101, 1, 1),
                                          (1, 127, 1, 1), (3, 24, 2, 1), (3, 9, 1, 7), (1, 2, 1, 1)])
def test_rows_and_positions(C, P, m, frames, dtype):
    rng = np.random.default_rng(P * 10 + m)
    total = sum(h * w * C for h, w in SIZES)
    pixels = rng.integers(0, 256, total, dtype=np.uint8)
    shapes, offsets, first, rows = pkg.patch_layout(SIZES, C, P, m)
    got, positions = pkg.patch_rows(torch.from_numpy(pixels).cuda(), shapes, offsets, first, rows, P, MEAN[:C], ISTD[:C], merge=m, frames=frames, dtype=dtype)
    check(got, positions, *reference(pixels, SIZES, C, P, m, frames))


def test_many_pictures_and_pixels_at_an_odd_address():
    """More pictures than the search asks at a time, some without a pixel; pixels that begin at any byte."""
    rng = np.random.default_rng(3)
    sizes = [(int(h), int(w)) if j % 7 else (0, int(w)) for j, (h, w) in enumerate(rng.integers(1, 40, (5000, 2)))]
    total = sum(h * w * 3 for h, w in sizes)
    for shift in (1, 2, 3):
        pixels = rng.integers(0, 256, total, dtype=np.uint8)
        held = torch.empty(total + 8, dtype=torch.uint8, device="cuda")
        held[shift:shift + total] = torch.from_numpy(pixels).cuda()
        shapes, offsets, first, rows = pkg.patch_layout(sizes, 3, 12)
        got, positions = pkg.patch_rows(held[shift:shift + total], shapes, offsets, first, rows, 12, MEAN, ISTD, dtype=torch.float32)
        check(got, positions, *reference(pixels, sizes, 3, 12, 1, 1))


def test_rows_without_a_picture_are_zero_and_pixels_that_are_not_there_are_not_read():
    sizes = [(20, 20), (30, 10)]
    pixels = torch.randint(0, 256, (20 * 20 * 3 + 30 * 10 * 3,), dtype=torch.uint8, device="cuda")
    shapes, offsets, first, rows = pkg.patch_layout(sizes, 3, 10)
    out = torch.full((rows + 5, 300), 7.0, dtype=torch.float16, device="cuda")
    positions = torch.full((3, rows + 5), 7, dtype=torch.int32, device="cuda")
    pkg.patch_rows(pixels, shapes, offsets, first, rows + 5, 10, MEAN, ISTD, out=out, positions=positions)
    assert not out[rows:].any() and not positions[:, rows:].any() and out[:rows].any()
    pkg.patch_rows(pixels[:-1], shapes, offsets, first, rows, 10, MEAN, ISTD, out=out[:rows], positions=positions[:, :rows].contiguous())
    assert not out[4:rows].any() and out[:4].any()            # the second picture lacks its last byte
    lost = offsets.clone()
    lost[1] = -5
    pkg.patch_rows(pixels, shapes, lost, first, rows, 10, MEAN, ISTD, out=out[:rows])
    assert not out[4:rows].any()
    few, _ = pkg.patch_rows(pixels, shapes, offsets, first, 3, 10, MEAN, ISTD, dtype=torch.float16)
    assert tuple(few.shape) == (3, 300)
    none, where = pkg.patch_rows(pixels, shapes, offsets, first, 0, 10, MEAN, ISTD)
    assert none.shape[0] == 0 and tuple(where.shape) == (3, 0)


def test_a_record(rgb_small):
    """Decode, layout from the record, rows: the pictures of the record at their sizes."""
    with pkg.pcr_open(rgb_small[0], 0) as r:
        pixels = r.decode_batch(10)
        layout = r.patch_layout(14, 2)
        got, positions = pkg.patch_rows(pixels, *layout, 14, MEAN, ISTD, merge=2, dtype=torch.bfloat16)
        sizes = [(h, w) for w, h, _, _ in (r.image_info(i) for i in range(r.n))]
        check(got, positions, *reference(pixels.cpu().numpy(), sizes, 3, 14, 2, 1))


def test_refusals():
    sizes = [(20, 20)]
    pixels = torch.zeros(1200, dtype=torch.uint8, device="cuda")
    shapes, offsets, first, rows = pkg.patch_layout(sizes, 3, 10)

    def call(**more):
        a = dict(pixels=pixels, shapes=shapes, offsets=offsets, first_rows=first, rows=rows, patch=10, mean=MEAN, inv_std=ISTD)
        a.update(more)
        return pkg.patch_rows(**a)
    call()
    for bad in (dict(pixels=pixels.cpu()), dict(pixels=pixels.float()), dict(shapes=shapes.long()), dict(offsets=offsets[:1]), dict(first_rows=first.int()),
                dict(mean=MEAN[:2]), dict(inv_std=ISTD[:1]), dict(rows=-1), dict(patch=0), dict(merge=0), dict(frames=0), dict(dtype=torch.float64),
                dict(out=torch.empty((rows, 299), dtype=torch.float16, device="cuda")), dict(positions=torch.empty((rows, 3), dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(patch=129, out=torch.empty((rows, 3 * 129 * 129), device="cuda")), dict(merge=17)):
        with pytest.raises(pkg.PcrError) as e:
            call(**bad)
        assert e.value.code == pkg.E_RANGE
