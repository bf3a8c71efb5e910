"""What group norm, position bias and dropout refuse before any device call, through the C entry points; the buckets of distances; and that none of their kernels spills."""
import ctypes
import math
import os
import subprocess

import pytest

import paper_1911_00472_amd as pkg

_i64, _i32, _vp, _f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


class Norm(ctypes.Structure):                              # pcr_group_norm
    _fields_ = [("x", _vp), ("x_image", _i64), ("x_pixel", _i64), ("out", _vp), ("out_image", _i64), ("out_pixel", _i64), ("grad", _vp), ("grad_image", _i64), ("grad_pixel", _i64),
                ("weight", _vp), ("bias", _vp), ("stats", _vp), ("weight_grad", _vp), ("bias_grad", _vp), ("images", _i64), ("pixels", _i64), ("channels", _i64), ("groups", _i32),
                ("activation", _i32), ("dtype", _i32), ("weight_dtype", _i32), ("eps", _f32), ("reserved", _f32)]


class Places(ctypes.Structure):                            # pcr_places
    _fields_ = [("position", _vp), ("axis_stride", _i64), ("batch_stride", _i64), ("token_stride", _i64), ("segment", _vp), ("segment_batch_stride", _i64), ("segment_token_stride", _i64)]


class Table(ctypes.Structure):                             # pcr_position_table
    _fields_ = [("query", Places), ("key", Places), ("map", _vp), ("table", _vp), ("values", _vp), ("value_batch", _i64), ("value_head", _i64), ("value_query", _i64), ("batch", _i64),
                ("heads", _i64), ("queries", _i64), ("keys", _i64), ("buckets", _i64), ("axes", _i32), ("reach", _i32), ("wide", _i32), ("dtype", _i32), ("table_dtype", _i32), ("reserved", _i32)]


class Dropout(ctypes.Structure):                           # pcr_dropout
    _fields_ = [("x", _vp), ("residual", _vp), ("out", _vp), ("seed", _vp), ("used", _vp), ("rows", _i64), ("dim", _i64), ("x_row", _i64), ("residual_row", _i64), ("out_row", _i64),
                ("p", ctypes.c_double), ("dtype", _i32), ("out_dtype", _i32), ("call", _i32), ("reserved", _i32)]


one = (ctypes.c_float * 4)()
at = ctypes.addressof(one)
by = ctypes.byref


def changed(of, **fields):
    for k, v in fields.items():
        setattr(of, k, v)
    return of


def norm(**fields):
    return changed(Norm(at, 16, 4, at, 16, 4, at, 16, 4, None, None, at, None, None, 1, 4, 4, 2, 0, 0, 0, 1e-5, 0.0), **fields)


def table(**fields):
    return changed(Table(Places(at, 4, 0, 1, None, 0, 0), Places(at, 4, 0, 1, None, 0, 0), at, at, at, 0, 16, 4, 1, 1, 4, 4, 3, 1, 1, 0, 0, 0, 0), **fields)


def dropout(**fields):
    return changed(Dropout(at, None, at, at, None, 2, 2, 2, 2, 2, 0.5, 0, 0, 0, 0), **fields)


def test_group_norm():
    L = pkg.lib()
    need = ctypes.c_size_t(0)
    for code, bad in ((pkg.E_ARG, dict(x=None)), (pkg.E_ARG, dict(out=None)), (pkg.E_ARG, dict(stats=None)), (pkg.E_ARG, dict(dtype=3)), (pkg.E_ARG, dict(weight_dtype=-1)),
                      (pkg.E_ARG, dict(dtype=1, weight_dtype=2)), (pkg.E_ARG, dict(activation=4)), (pkg.E_ARG, dict(activation=-1)), (pkg.E_RANGE, dict(groups=3)), (pkg.E_RANGE, dict(groups=0)),
                      (pkg.E_RANGE, dict(channels=0)), (pkg.E_RANGE, dict(channels=16386)), (pkg.E_RANGE, dict(channels=16384, groups=8192)), (pkg.E_RANGE, dict(images=-1)), (pkg.E_RANGE, dict(pixels=-1)),
                      (pkg.E_RANGE, dict(images=2 ** 31)), (pkg.E_RANGE, dict(pixels=2 ** 41))):
        assert L.pcr_group_norm_forward(0, by(norm(**bad)), at, 1 << 40, None) == code, bad
        assert L.pcr_group_norm_backward(0, by(norm(**bad)), at, 1 << 40, None) == code, bad
    for eps in (-1.0, math.nan, math.inf):
        assert L.pcr_group_norm_forward(0, by(norm(eps=eps)), at, 1 << 40, None) == pkg.E_RANGE
    assert L.pcr_group_norm_backward(0, by(norm(grad=None)), at, 1 << 40, None) == pkg.E_ARG
    assert L.pcr_group_norm_forward(0, None, at, 64, None) == pkg.E_ARG and L.pcr_group_norm_backward(0, None, at, 64, None) == pkg.E_ARG
    large = dict(images=3, pixels=1 << 24)
    for backward, f in ((0, L.pcr_group_norm_forward), (1, L.pcr_group_norm_backward)):
        assert L.pcr_group_norm_workspace(by(norm(**large)), backward, by(need)) == pkg.OK and need.value > 0
        assert f(0, by(norm(**large)), None, need.value, None) == pkg.E_ARG
        assert f(0, by(norm(**large)), at, need.value - 1, None) == pkg.E_RANGE
        assert f(0, by(norm(**large)), (at + 15) // 16 * 16 + 8, need.value, None) == pkg.E_ARG          # (working memory not at a multiple of 16)
    assert L.pcr_group_norm_workspace(None, 0, by(need)) == pkg.E_ARG and L.pcr_group_norm_workspace(by(norm()), 0, None) == pkg.E_ARG
    assert L.pcr_group_norm_workspace(by(norm(groups=3)), 0, by(need)) == pkg.E_RANGE
    assert L.pcr_group_norm_forward(0, by(norm(images=0, x=None, out=None, stats=None)), None, 0, None) == pkg.OK


def test_rows_of_many_small_pictures():
    """Working memory for channels' sums goes by workgroups, not by pictures, and covers pictures that do not divide evenly."""
    need, L = ctypes.c_size_t(0), pkg.lib()
    for images in (2048, 4097, 100000, 2 ** 24 + 3):
        assert L.pcr_group_norm_workspace(by(norm(images=images, pixels=4, channels=32, groups=4, x_pixel=32, out_pixel=32, grad_pixel=32, x_image=128, out_image=128, grad_image=128, dtype=2, weight_dtype=2)),
                                          1, by(need)) == pkg.OK
        rows, rest = divmod(need.value, 32 * 8)
        assert rest == 0 and images / 512 <= rows <= images, (images, rows)


def test_position_bias():
    L = pkg.lib()
    need = ctypes.c_size_t(0)

    def both(t):
        return L.pcr_position_bias(0, by(t), None), L.pcr_position_bias_backward(0, by(t), at, at, 1 << 40, None), L.pcr_position_bias_workspace(by(t), by(need))
    for code, bad in ((pkg.E_ARG, dict(dtype=3)), (pkg.E_ARG, dict(map=None)), (pkg.E_ARG, dict(values=None)), (pkg.E_ARG, dict(query=Places())), (pkg.E_ARG, dict(key=Places())),
                      (pkg.E_ARG, dict(query=Places(at, 4, 0, 1, at, 0, 1))), (pkg.E_RANGE, dict(axes=0)), (pkg.E_RANGE, dict(axes=5)), (pkg.E_RANGE, dict(reach=-1)), (pkg.E_RANGE, dict(reach=2 ** 24 + 1)),
                      (pkg.E_RANGE, dict(buckets=0)), (pkg.E_RANGE, dict(buckets=2 ** 24 + 1)), (pkg.E_RANGE, dict(heads=-1)), (pkg.E_RANGE, dict(heads=65536)), (pkg.E_RANGE, dict(batch=-1)),
                      (pkg.E_RANGE, dict(queries=2 ** 31)), (pkg.E_RANGE, dict(keys=-1)), (pkg.E_RANGE, dict(batch=2 ** 30, queries=2 ** 20, keys=2))):
        assert both(table(**bad)) == (code,) * 3, bad
    assert L.pcr_position_bias(0, by(table(table=None)), None) == pkg.E_ARG and L.pcr_position_bias(0, by(table(table_dtype=4)), None) == pkg.E_ARG
    assert L.pcr_position_bias(0, by(table(dtype=1, table_dtype=2)), None) == pkg.E_ARG
    assert L.pcr_position_bias(0, None, None) == pkg.E_ARG and L.pcr_position_bias_workspace(None, by(need)) == pkg.E_ARG and L.pcr_position_bias_workspace(by(table()), None) == pkg.E_ARG
    long = dict(queries=1000, keys=1000)
    assert L.pcr_position_bias_workspace(by(table(**long)), by(need)) == pkg.OK and need.value > 0
    assert L.pcr_position_bias_backward(0, by(table(**long)), None, at, need.value, None) == pkg.E_ARG
    assert L.pcr_position_bias_backward(0, by(table(**long)), at, None, need.value, None) == pkg.E_ARG
    assert L.pcr_position_bias_backward(0, by(table(**long)), at, at, need.value - 1, None) == pkg.E_RANGE
    assert L.pcr_position_bias_backward(0, by(table(**long)), at, (at + 15) // 16 * 16 + 8, need.value, None) == pkg.E_ARG
    assert L.pcr_position_bias(0, by(table(keys=0, query=Places(), key=Places(), map=None, values=None)), None) == pkg.OK


def test_dropout():
    L = pkg.lib()
    for code, bad in ((pkg.E_ARG, dict(x=None)), (pkg.E_ARG, dict(out=None)), (pkg.E_ARG, dict(seed=None)), (pkg.E_ARG, dict(dtype=3)), (pkg.E_ARG, dict(out_dtype=-1)), (pkg.E_ARG, dict(dtype=1, out_dtype=2)),
                      (pkg.E_RANGE, dict(rows=-1)), (pkg.E_RANGE, dict(dim=-1)), (pkg.E_RANGE, dict(p=-0.1)), (pkg.E_RANGE, dict(p=1.5)), (pkg.E_RANGE, dict(p=math.nan)), (pkg.E_RANGE, dict(call=-1)),
                      (pkg.E_RANGE, dict(call=65536)), (pkg.E_RANGE, dict(rows=2 ** 40, dim=2 ** 11)), (pkg.E_RANGE, dict(rows=2 ** 62, dim=2 ** 62))):
        assert L.pcr_dropout_add(0, by(dropout(**bad)), None) == code, bad
    assert L.pcr_dropout_add(0, None, None) == pkg.E_ARG
    assert L.pcr_dropout_add(0, by(dropout(rows=0, x=None, out=None, seed=None)), None) == pkg.OK


def test_buckets_of_windows_and_lines():
    m, n = pkg.position_buckets((3, 4), device="cpu")          # a window of 3 x 4: a bucket for every difference, rows first
    assert n == 5 * 7 and m.shape == (2, 7)
    for r in range(-2, 3):
        for c in range(-3, 4):
            assert int(m[0, 3 + r] + m[1, 3 + c]) == (r + 2) * 7 + c + 3
    assert m[0].tolist() == [0, 0, 7, 14, 21, 28, 28]          # (a distance past the last bucket's counts as that)
    m, n = pkg.position_buckets(8, 8, 128, device="cpu")
    assert n == 31 and m.shape == (1, 257)
    for d in range(-128, 129):
        x = abs(d)
        side = x if x < 8 else min(15, 8 + sum(x >= b for b in (8 * 2 ** 0.5, 16, 16 * 2 ** 0.5, 32, 32 * 2 ** 0.5, 64, 64 * 2 ** 0.5)))
        assert int(m[0, 128 + d]) == 15 + (side if d > 0 else -side), d
    m, n = pkg.position_buckets(4, 3, 32, one_sided=True, device="cpu")
    assert n == 7 and m[0, 32:].tolist() == [0] * 33 and m[0, :33].tolist()[::-1] == [0, 1, 2, 3] + [4] * 4 + [5] * 8 + [6] * 17
    m, n = pkg.position_buckets((1, 2, 3), (0, 2, 0), (0, 8, 0), device="cpu")
    assert n == 1 * 7 * 5 and m.shape == (3, 17) and not m[0].any()
    assert pkg.position_buckets(1, device="cpu")[0].tolist() == [[0]]
    for bad in ((0,), (4, -1), (4, 2, 4), ((1,) * 5,), ((3, 4), (1, 1, 1), 9), (5000, 0, 0), ((200, 200, 200),)):
        if bad == (5000, 0, 0):
            assert pkg.position_buckets(*bad, device="cpu")[1] == 9999
            continue
        with pytest.raises(ValueError):
            pkg.position_buckets(*bad, device="cpu")


def test_no_kernel_spills_to_scratch_memory(tmp_path):
    from paper_1911_00472_amd import build
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    sources = [build.SRC_LAYERS, build.SRC_NORM_HELD, build.SRC_NORM_BACK_HELD]
    listings = [tmp_path / (os.path.basename(s) + ".s") for s in sources]
    running = [subprocess.Popen([hipcc] + flags + ["-S", "--cuda-device-only", "-o", str(to), s], stderr=subprocess.DEVNULL) for s, to in zip(sources, listings)]
    assert [p.wait() for p in running] == [0] * len(sources)
    sizes = [line.split()[-1] for to in listings for line in to.read_text().splitlines() if ".amdhsa_private_segment_fixed_size" in line]
    assert len(sizes) > 30 and all(s == "0" for s in sizes), sizes
