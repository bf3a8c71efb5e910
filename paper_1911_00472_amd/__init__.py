"""MI355X (gfx950) decoder for Progressive Compressed Records: C-ABI library in csrc/ built to
libpcr.so, plus a thin ctypes binding with the same entry-point names (binding.py; train.py for the operators behind the decode)."""
from .binding import (E_ARG, E_DEVICE, E_FORMAT, E_NOMEM, E_RANGE, E_TRUNCATED, E_UNSUPPORTED, LIB_PATH, NUM_STAGES, OK,
                      STAGE_NAMES, SYMBOLS, Loader, PcrError, Record, lib, pcr_open, pcr_open_device, prefix_length,
                      probe_scalar_issue_rate, record_write, record_write_indexed, scan_ends, transcode_files, transcode_progressive, transcode_symbol_counts)

_TRAIN = ("patch_layout", "patch_rows", "axis_frequencies", "rotate_axes", "norm_rotate", "norm_rotate_backward", "distill_forward", "distill_backward",
          "distill_step", "distill_loss")


def _deferred(name):
    def call(*args, **kwargs):
        from . import train
        return getattr(train, name)(*args, **kwargs)
    call.__name__ = call.__qualname__ = name
    return call


def __getattr__(name):
    """The operators of train.py, with PyTorch, when the first of them is asked for.  Where they cannot be had (nothing is built, no PyTorch) the names
    are there all the same, for `import *`, and a call says what is missing."""
    if name in _TRAIN:
        try:
            from . import train
        except (ImportError, OSError, RuntimeError):
            return _deferred(name)
        for n in _TRAIN:
            globals()[n] = getattr(train, n)
        return globals()[name]
    raise AttributeError("module %r has no attribute %r" % (__name__, name))


__all__ = [*_TRAIN, "Record", "Loader", "prefix_length", "scan_ends", "record_write", "record_write_indexed", "transcode_progressive", "transcode_symbol_counts", "transcode_files", "pcr_open", "pcr_open_device", "probe_scalar_issue_rate", "PcrError", "lib", "SYMBOLS", "LIB_PATH", "STAGE_NAMES", "NUM_STAGES",
           "OK", "E_ARG", "E_FORMAT", "E_TRUNCATED", "E_UNSUPPORTED", "E_RANGE", "E_NOMEM", "E_DEVICE"]
