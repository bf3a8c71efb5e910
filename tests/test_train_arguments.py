"""What the operators behind the decode refuse before any device call, through the C entry points; and that none of their kernels spills."""
import ctypes
import os
import subprocess

import pytest

import paper_1911_00472_amd as pkg

_i64, _i32, _vp, _f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_float


class Heads(ctypes.Structure):                             # pcr_heads
    _fields_ = [("in_", _vp), ("in_batch", _i64), ("in_token", _i64), ("in_head", _i64), ("out", _vp), ("out_batch", _i64), ("out_token", _i64), ("out_head", _i64),
                ("grad", _vp), ("grad_batch", _i64), ("grad_token", _i64), ("grad_head", _i64), ("weight", _vp), ("weight_grad", _vp), ("heads", _i64)]


class Rotation(ctypes.Structure):                          # pcr_rotation
    _fields_ = [("position", _vp), ("axis_stride", _i64), ("batch_stride", _i64), ("token_stride", _i64), ("frequency", _vp), ("axis", _vp), ("batch", _i64), ("tokens", _i64),
                ("wide", _i32), ("axes", _i32), ("dim", _i32), ("pairs", _i32), ("adjacent", _i32), ("reserved", _i32)]


class Distill(ctypes.Structure):                           # pcr_distill
    _fields_ = [("logits", _vp), ("row_stride", _i64), ("top_index", _vp), ("top_logits", _vp), ("labels", _vp), ("rows", _i64), ("classes", _i64), ("top", _i32), ("dtype", _i32),
                ("top_dtype", _i32), ("index_wide", _i32), ("temperature", _f32), ("distill_part", _f32), ("label_part", _f32), ("reserved", _f32)]


def test_null_pointers_and_sizes_out_of_range():
    L = pkg.lib()
    one = (ctypes.c_float * 3)(1, 1, 1)
    at = ctypes.cast(one, ctypes.c_void_p)
    patch = [0, at, 12, at, at, at, 1, 1, 2, 1, 1, 3, one, one, 0, at, None, None]

    def with_(args, **changed):
        return [changed.get("a%d" % i, v) for i, v in enumerate(args)]
    for code, changed in ((pkg.E_ARG, dict(a1=None)), (pkg.E_ARG, dict(a3=None)), (pkg.E_ARG, dict(a4=None)), (pkg.E_ARG, dict(a5=None)), (pkg.E_ARG, dict(a12=None)), (pkg.E_ARG, dict(a13=None)),
                          (pkg.E_ARG, dict(a14=3)), (pkg.E_ARG, dict(a15=None)), (pkg.E_RANGE, dict(a6=-1)), (pkg.E_RANGE, dict(a7=-1)), (pkg.E_RANGE, dict(a8=0)), (pkg.E_RANGE, dict(a8=129)),
                          (pkg.E_RANGE, dict(a9=0)), (pkg.E_RANGE, dict(a10=0)), (pkg.E_RANGE, dict(a11=2))):
        assert L.pcr_patch_rows(*with_(patch, **changed)) == code, changed
    assert L.pcr_patch_rows(*with_(patch, a7=0)) == pkg.OK                      # no rows: nothing to do

    def rotation(**changed):
        r = Rotation(at, 1, 1, 1, at, at, 1, 1, 0, 1, 8, 4, 0, 0)
        for k, v in changed.items():
            setattr(r, k, v)
        return r

    def heads(**changed):
        h = Heads(at, 0, 0, 0, at, 0, 0, 0, at, 0, 0, 0, None, None, 1)
        for k, v in changed.items():
            setattr(h, k, v)
        return h
    by = ctypes.byref
    assert L.pcr_rotate_axes(0, None, by(heads()), by(rotation()), 0, 0, None) == pkg.E_ARG
    assert L.pcr_rotate_axes(0, by(heads()), None, by(rotation()), 0, 0, None) == pkg.E_ARG
    assert L.pcr_rotate_axes(0, by(heads()), by(heads()), None, 0, 0, None) == pkg.E_ARG
    assert L.pcr_rotate_axes(0, by(heads()), by(heads()), by(rotation()), 0, 5, None) == pkg.E_ARG
    for bad in (dict(dim=0), dict(dim=513), dict(pairs=5), dict(pairs=-1), dict(axes=0), dict(axes=5), dict(batch=-1), dict(tokens=-1), dict(tokens=2 ** 31), dict(batch=2 ** 20, tokens=2 ** 20)):
        assert L.pcr_rotate_axes(0, by(heads()), by(heads()), by(rotation(**bad)), 0, 0, None) == pkg.E_RANGE, bad
    for bad in (dict(position=None), dict(frequency=None), dict(axis=None)):
        assert L.pcr_rotate_axes(0, by(heads()), by(heads()), by(rotation(**bad)), 0, 0, None) == pkg.E_ARG, bad
    for bad in (dict(in_=None), dict(out=None)):
        assert L.pcr_norm_rotate(0, by(heads()), by(heads(**bad)), by(rotation()), 1e-6, 0, 0, None) == pkg.E_ARG, bad
    assert L.pcr_norm_rotate(0, by(heads(heads=-1)), by(heads()), by(rotation()), 1e-6, 0, 0, None) == pkg.E_RANGE
    assert L.pcr_norm_rotate(0, by(heads()), by(heads()), by(rotation()), 1e-6, 1, 2, None) == pkg.E_ARG          # weights of a third type
    assert L.pcr_norm_rotate_backward(0, by(heads(grad=None)), by(heads()), by(rotation()), 1e-6, 0, 0, None, 0, None) == pkg.E_ARG
    need = ctypes.c_size_t(0)
    assert L.pcr_norm_rotate_workspace(100, 8, by(need)) == pkg.OK and need.value > 0
    assert L.pcr_norm_rotate_workspace(-1, 8, by(need)) == pkg.E_RANGE and L.pcr_norm_rotate_workspace(1, 8, None) == pkg.E_ARG
    asks = heads(weight_grad=ctypes.addressof(one))
    assert L.pcr_norm_rotate_backward(0, by(asks), by(heads()), by(rotation()), 1e-6, 0, 0, None, 0, None) == pkg.E_ARG
    assert L.pcr_norm_rotate_backward(0, by(asks), by(heads()), by(rotation()), 1e-6, 0, 0, at, 8, None) == pkg.E_RANGE

    def distill(**changed):
        d = Distill(at, 10, at, at, None, 2, 10, 3, 0, 0, 0, 1.0, 1.0, 0.0, 0.0)
        for k, v in changed.items():
            setattr(d, k, v)
        return d
    for code, bad in ((pkg.E_ARG, dict(logits=None)), (pkg.E_ARG, dict(top_index=None)), (pkg.E_ARG, dict(top_logits=None)), (pkg.E_ARG, dict(dtype=3)), (pkg.E_ARG, dict(top_dtype=-1)), (pkg.E_RANGE, dict(rows=-1)),
                      (pkg.E_RANGE, dict(classes=0)), (pkg.E_RANGE, dict(classes=2 ** 31)), (pkg.E_RANGE, dict(top=0)), (pkg.E_RANGE, dict(top=1025)), (pkg.E_RANGE, dict(temperature=0.0)),
                      (pkg.E_RANGE, dict(temperature=float("nan"))), (pkg.E_RANGE, dict(distill_part=float("inf"))), (pkg.E_RANGE, dict(label_part=float("nan")))):
        d = distill(**bad)
        assert L.pcr_distill_forward(0, by(d), at, at, None, 0, None) == code, bad
        assert L.pcr_distill_backward(0, by(d), at, at, at, 10, None) == code, bad
        assert L.pcr_distill_step(0, by(d), at, at, at, 10, None, 0, None) == code, bad
    assert L.pcr_distill_forward(0, None, at, at, None, 0, None) == pkg.E_ARG
    assert L.pcr_distill_forward(0, by(distill()), None, at, None, 0, None) == pkg.E_ARG
    assert L.pcr_distill_backward(0, by(distill()), None, at, at, 10, None) == pkg.E_ARG
    assert L.pcr_distill_step(0, by(distill()), at, at, None, 10, None, 0, None) == pkg.E_ARG
    wide = distill(rows=1, classes=10 ** 6)
    assert L.pcr_distill_workspace(1, 10 ** 6, by(need)) == pkg.OK and need.value > 0
    assert L.pcr_distill_forward(0, by(wide), at, at, None, 0, None) == pkg.E_ARG
    assert L.pcr_distill_step(0, by(wide), at, at, at, 10 ** 6, at, 8, None) == pkg.E_RANGE
    assert L.pcr_distill_workspace(-1, 10, by(need)) == pkg.E_RANGE and L.pcr_distill_workspace(1, 10, None) == pkg.E_ARG


@pytest.mark.parametrize("source", ["SRC_TRAIN", "SRC_DISTILL"])
def test_no_kernel_spills_to_scratch_memory(tmp_path, source):
    from paper_1911_00472_amd import build
    asm = tmp_path / "kernels.s"
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.check_call([hipcc] + flags + ["-S", "--cuda-device-only", "-o", str(asm), getattr(build, source)], stderr=subprocess.DEVNULL)
    sizes = [line.split()[-1] for line in asm.read_text().splitlines() if ".amdhsa_private_segment_fixed_size" in line]
    assert len(sizes) > 30 and all(s == "0" for s in sizes), sizes
