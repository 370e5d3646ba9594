"""ctypes binding of libaug.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI declared in
include/aug.h.  PyTorch tensors supply device memory and the stream.  There is
no CPU fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libaug.so")

AUG_OK = 0
AUG_ERR_INVALID_ARG = -1
AUG_ERR_UNSUPPORTED = -2
AUG_ERR_NOMEM = -3
AUG_ERR_HIP = -4

EXPORTS = ("aug_create", "aug_destroy", "aug_last_error", "aug_frame_count", "aug_feature_dim", "aug_rir_batch",
           "aug_rir_mics_batch",
           "aug_convolve_mix_batch", "aug_vtlp_mel_batch", "aug_vtlp_mel_batch_static", "aug_vtlp_resynth_batch",
           "aug_pipeline_batch",
           "aug_rms_norm_batch", "aug_rms_norm_backward_batch",
           "aug_short_conv_batch", "aug_short_conv_backward_batch", "aug_short_conv_step",
           "aug_scan_batch", "aug_scan_backward_batch", "aug_scan_step",
           "aug_profile_enable", "aug_profile_read", "aug_rir_visited_images")

FEATURE_KINDS = {"power": 0, "log": 1, "mfcc": 2}      # AUG_FEAT_*

STAGES = ("rir", "rir_spectrum", "convolve", "mix", "mel", "other", "vtlp", "norm", "short_conv", "scan")

ACTIVATIONS = {"none": 0, "silu": 1}


class VtlpCfg(ctypes.Structure):
    """Mirror of aug_vtlp_cfg."""
    _fields_ = [("win", ctypes.c_int), ("hop", ctypes.c_int), ("nfft", ctypes.c_int)]


# The C structs of the operators on feature rows as arrays of their fields, which is the cheapest way to fill them: a call for a few
# streams takes the GPU four microseconds.
ROWS = ctypes.c_int64 * 2               # aug_rows: data, ld
SCAN_IN = ctypes.c_int64 * 13           # aug_scan_in: u, delta, b, c, z (aug_rows each), a, skip, delta_bias
SCAN_GRAD = ctypes.c_int64 * 13         # aug_scan_grad: du, ddelta, db, dc, dz, da, dskip, ddelta_bias
SHORT_CONV_CFG = ctypes.c_int * 4       # aug_short_conv_cfg: dtype, dim, taps, silu
SCAN_CFG = ctypes.c_int * 5             # aug_scan_cfg: dtype, dim, n_state, n_group, softplus


class NormCfg(ctypes.Structure):
    """Mirror of aug_norm_cfg."""
    _fields_ = [("dtype", ctypes.c_int), ("dim", ctypes.c_int), ("eps", ctypes.c_float), ("q_block", ctypes.c_int)]


class AugError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libaug error {code}: {message}")
        self.code = code


class FrontendCfg(ctypes.Structure):
    """Mirror of aug_frontend_cfg."""
    _fields_ = [("fs", ctypes.c_float), ("win", ctypes.c_int), ("hop", ctypes.c_int),
                ("nfft", ctypes.c_int), ("n_mel", ctypes.c_int), ("f_lo", ctypes.c_float),
                ("f_hi", ctypes.c_float), ("power", ctypes.c_float), ("feature", ctypes.c_int),
                ("n_ceps", ctypes.c_int), ("log_floor", ctypes.c_float)]

    @classmethod
    def of(cls, fe) -> "FrontendCfg":
        return cls(float(fe.fs), int(fe.win), int(fe.hop), int(fe.nfft), int(fe.n_mel),
                   float(fe.f_lo), float(fe.f_hi), float(fe.power),
                   FEATURE_KINDS[getattr(fe, "feature", "power")], int(getattr(fe, "n_ceps", 0)),
                   float(getattr(fe, "log_floor", 1e-10)))


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libaug.so (built in-tree by build.py); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build the HIP library first "
            "(python -m paper_1912_11040_amd.build); there is no CPU fallback")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci, cf, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_int64
    p_i64 = ctypes.POINTER(ctypes.c_int64)
    p_cfg = ctypes.POINTER(FrontendCfg)
    lib.aug_create.argtypes = [ctypes.POINTER(vp), ci, vp]
    lib.aug_create.restype = ci
    lib.aug_destroy.argtypes = [vp]
    lib.aug_destroy.restype = ci
    lib.aug_last_error.argtypes = [vp]
    lib.aug_last_error.restype = ctypes.c_char_p
    lib.aug_frame_count.argtypes = [i64, ci, ci]
    lib.aug_frame_count.restype = i64
    lib.aug_feature_dim.argtypes = [p_cfg]
    lib.aug_feature_dim.restype = ci
    lib.aug_rir_batch.argtypes = [vp, ci, vp, ci, cf, cf, vp, vp]
    lib.aug_rir_batch.restype = ci
    lib.aug_rir_mics_batch.argtypes = [vp, ci, ci, vp, vp, ci, cf, cf, vp, vp]
    lib.aug_rir_mics_batch.restype = ci
    lib.aug_convolve_mix_batch.argtypes = [vp, ci, p_i64, vp, ci, vp, vp, ci, vp, vp, vp]
    lib.aug_convolve_mix_batch.restype = ci
    lib.aug_vtlp_mel_batch.argtypes = [vp, ci, p_i64, vp, vp, p_cfg, p_i64, vp]
    lib.aug_vtlp_mel_batch.restype = ci
    lib.aug_vtlp_mel_batch_static.argtypes = [vp, ci, p_i64, vp, vp, p_cfg, p_i64, vp]
    lib.aug_vtlp_mel_batch_static.restype = ci
    lib.aug_vtlp_resynth_batch.argtypes = [vp, ci, p_i64, vp, vp, ctypes.POINTER(VtlpCfg), vp]
    lib.aug_vtlp_resynth_batch.restype = ci
    lib.aug_pipeline_batch.argtypes = [vp, ci, p_i64, vp, ci, vp, vp, ci, cf, cf, vp, vp, p_cfg,
                                       p_i64, vp, vp, vp, vp]
    lib.aug_pipeline_batch.restype = ci
    lib.aug_rms_norm_batch.argtypes = [vp, i64] + [vp] * 9
    lib.aug_rms_norm_backward_batch.argtypes = [vp, i64] + [vp] * 8
    lib.aug_short_conv_batch.argtypes = [vp, ci] + [vp] * 9
    lib.aug_short_conv_backward_batch.argtypes = [vp, ci] + [vp] * 11
    lib.aug_short_conv_step.argtypes = [vp, ci] + [vp] * 7
    lib.aug_scan_batch.argtypes = [vp, ci] + [vp] * 7
    lib.aug_scan_backward_batch.argtypes = [vp, ci] + [vp] * 7
    lib.aug_scan_step.argtypes = [vp, ci] + [vp] * 5
    for name in EXPORTS:
        if name.startswith(("aug_rms_norm", "aug_short_conv", "aug_scan")):
            getattr(lib, name).restype = ci
    lib.aug_rir_visited_images.argtypes = [vp, ci, vp, ci, cf, cf, vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.aug_rir_visited_images.restype = ci
    lib.aug_profile_enable.argtypes = [vp, ci]
    lib.aug_profile_enable.restype = ci
    lib.aug_profile_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32)]
    lib.aug_profile_read.restype = ci
    _lib = lib
    return lib


def aug_frame_count(n_samples: int, win: int, hop: int) -> int:
    return int(load_library().aug_frame_count(int(n_samples), int(win), int(hop)))


def _host_i64(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int64))


def _ptr(t, dtype=None):
    """Device address of a contiguous CUDA/HIP torch tensor (None -> NULL)."""
    if t is None:
        return None
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("expected a torch tensor in device memory")
    if not t.is_contiguous():
        raise ValueError("device tensors must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected dtype {dtype}, got {t.dtype}")
    return ctypes.c_void_p(t.data_ptr())


def _numel(t) -> int:
    return 0 if t is None else int(t.numel())


def _need(name: str, t, count: int, exact: bool = False):
    """Raise ValueError unless tensor `t` holds at least (exactly) `count` elements; None counts as empty."""
    have = _numel(t)
    if (have != count) if exact else (have < count):
        raise ValueError(f"{name} holds {have} elements, the call needs {'exactly' if exact else 'at least'} {count}")


# Element counts that the C ABI takes on trust (it sees bare addresses): checked here, on the host, before
# anything is launched.  An undersized output would otherwise be written past its end by a kernel.

def check_offsets_pair(off: np.ndarray, foff: Optional[np.ndarray] = None):
    if off.ndim != 1 or len(off) < 1:
        raise ValueError("offsets must be a one-dimensional array of n_utt + 1 entries")
    if foff is not None and len(foff) != len(off):
        raise ValueError(f"frame_offsets has {len(foff)} entries, offsets has {len(off)}")


def check_rir_sizes(geom, rir_len: int, rir_out, tap_count_out, mics=None, n_mic: int = 1):
    if _numel(geom) % 10:
        raise ValueError("geom must hold 10 values per response")
    n_rir = _numel(geom) // 10
    n_mic, rir_len = max(int(n_mic), 0), max(int(rir_len), 0)      # the library refuses the negative ones itself
    if mics is not None:
        _need("mics", mics, n_rir * n_mic * 3)
    _need("rir_out", rir_out, n_rir * n_mic * rir_len)
    if tap_count_out is not None:
        _need("tap_count_out", tap_count_out, n_rir * n_mic * rir_len)


def check_mix_sizes(off: np.ndarray, speech, n_noise: int, noise, snr_db, gains_out=None):
    n_utt, total = len(off) - 1, int(off[-1])
    _need("speech", speech, total)
    _need("noise", noise, n_noise * total)
    _need("snr_db", snr_db, n_utt * n_noise)
    if gains_out is not None:
        _need("gains_out", gains_out, n_utt * n_noise)


def check_convolve_mix_sizes(off: np.ndarray, speech, n_noise: int, noise, rir, rir_len: int, snr_db, mixed_out,
                             gains_out=None):
    check_offsets_pair(off)
    check_mix_sizes(off, speech, n_noise, noise, snr_db, gains_out)
    _need("rir", rir, (len(off) - 1) * (1 + n_noise) * int(rir_len))
    _need("mixed_out", mixed_out, int(off[-1]))


def check_mel_sizes(off: np.ndarray, foff: np.ndarray, wave, alpha, feats_out, feature_dim: int):
    check_offsets_pair(off, foff)
    _need("wave", wave, int(off[-1]))
    _need("alpha", alpha, len(off) - 1)
    _need("feats_out", feats_out, int(foff[-1]) * int(feature_dim))


def check_pipeline_sizes(off: np.ndarray, foff: np.ndarray, speech, n_noise: int, noise, geom, rir_len: int,
                         snr_db, alpha, feature_dim: int, feats_out, rir_out=None, mixed_out=None, gains_out=None):
    check_offsets_pair(off, foff)
    n_utt = len(off) - 1
    check_mix_sizes(off, speech, n_noise, noise, snr_db, gains_out)
    _need("geom", geom, n_utt * (1 + n_noise) * 10, exact=True)
    _need("alpha", alpha, n_utt)
    _need("feats_out", feats_out, int(foff[-1]) * int(feature_dim))
    if rir_out is not None:
        _need("rir_out", rir_out, n_utt * (1 + n_noise) * int(rir_len))
    if mixed_out is not None:
        _need("mixed_out", mixed_out, int(off[-1]))


def check_resynth_sizes(off: np.ndarray, wave, alpha, wave_out):
    check_offsets_pair(off)
    _need("wave", wave, int(off[-1]))
    _need("alpha", alpha, len(off) - 1)
    _need("wave_out", wave_out, int(off[-1]))


# ---- operators on feature rows: shapes, which the C ABI sees as a leading dimension and a count only ----

@functools.lru_cache(maxsize=None)
def _element_types():
    import torch
    return {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}      # AUG_F32, AUG_BF16, AUG_F16


def _element_type(t) -> int:
    try:
        return _element_types()[t.dtype]
    except KeyError:
        raise TypeError(f"expected float32, bfloat16 or float16, got {t.dtype}") from None


def check_matrix(name: str, t, n_rows: int, width: int, dtype) -> int:
    """Raise unless `t` has at least n_rows rows of exactly `width` columns next to each other; its leading dimension."""
    shape = t.shape
    if len(shape) != 2 or shape[0] < n_rows or shape[1] != width:
        raise ValueError(f"{name} is {tuple(shape)}, the call needs {n_rows} rows of {width}")
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
    down, across = t.stride()
    if across != 1 and width > 1:
        raise ValueError(f"the columns of {name} are not next to each other")
    if shape[0] <= 1:
        return width
    if down < width:
        raise ValueError(f"the rows of {name} overlap")
    return down


def check_array(name: str, t, count: int, dtype):
    """Raise unless `t` is a contiguous tensor of exactly `count` elements."""
    if t.numel() != count:
        raise ValueError(f"{name} holds {t.numel()} elements, the call needs exactly {count}")
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def check_row_offsets(off: np.ndarray, lengths: Optional[np.ndarray] = None) -> int:
    """The rows that the sequences of a call reach."""
    check_offsets_pair(off)
    if lengths is None:
        return int(off[-1])
    if lengths.ndim != 1 or len(lengths) != len(off) - 1:
        raise ValueError(f"row_lengths has {lengths.size} entries, row_offsets has {len(off)}")
    return int((off[:-1] + lengths).max(initial=0))


def _two_dimensions(name: str, t):
    if len(t.shape) != 2:
        raise ValueError(f"{name} must have two dimensions")
    return t.shape


class Augmenter:
    """One library context bound to a device and a stream (torch's current stream by default)."""

    def __init__(self, device: int = 0, stream=None, check_sizes: bool = True):
        """check_sizes=False skips the host-side element-count checks of the tensors (the library still
        validates everything it can see: nulls, sizes, offsets)."""
        import torch
        self._lib = load_library()
        self._check_sizes = bool(check_sizes)
        self._f32 = torch.float32
        if stream is None:
            stream = torch.cuda.current_stream(device)
        self.stream = stream
        self.device = device
        handle = ctypes.c_void_p()
        rc = self._lib.aug_create(ctypes.byref(handle), int(device), ctypes.c_void_p(stream.cuda_stream))
        if rc != AUG_OK:
            raise AugError(rc, "aug_create failed")
        self._h = handle

    def close(self):
        if getattr(self, "_h", None):
            self._lib.aug_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _check(self, rc: int):
        if rc != AUG_OK:
            raise AugError(rc, self._lib.aug_last_error(self._h).decode())

    def aug_profile_enable(self, on: bool):
        self._check(self._lib.aug_profile_enable(self._h, int(bool(on))))

    def aug_profile_read(self):
        """Wait for the stream; {stage: (total ms, launches)} since the last read."""
        ms = (ctypes.c_float * len(STAGES))()
        n = (ctypes.c_int32 * len(STAGES))()
        self._check(self._lib.aug_profile_read(self._h, ms, n))
        return {name: (float(ms[i]), int(n[i])) for i, name in enumerate(STAGES)}

    # ---- the four entry points, same names as the C ABI ----

    def aug_rir_batch(self, geom, rir_len: int, fs: float, c: float, rir_out, tap_count_out=None):
        import torch
        if self._check_sizes:
            check_rir_sizes(geom, rir_len, rir_out, tap_count_out)
        n_rir = int(geom.numel() // 10) if geom is not None else 0
        self._check(self._lib.aug_rir_batch(
            self._h, n_rir, _ptr(geom, torch.float32), int(rir_len), float(fs), float(c),
            _ptr(rir_out, torch.float32), _ptr(tap_count_out, torch.int32)))

    def aug_rir_visited_images(self, geom, rir_len: int, fs: float, c: float, rir_out) -> int:
        """Images the amplitude kernel walks for these rooms (measurement helper; waits for the stream)."""
        import torch
        if self._check_sizes:
            check_rir_sizes(geom, rir_len, rir_out, None)
        n_rir = int(geom.numel() // 10) if geom is not None else 0
        n = ctypes.c_uint64(0)
        self._check(self._lib.aug_rir_visited_images(
            self._h, n_rir, _ptr(geom, torch.float32), int(rir_len), float(fs), float(c),
            _ptr(rir_out, torch.float32), ctypes.byref(n)))
        return int(n.value)

    def aug_rir_mics_batch(self, geom, mics, rir_len: int, fs: float, c: float, rir_out, tap_count_out=None,
                           n_mic: Optional[int] = None):
        """geom [n_rir][10], mics [n_rir][n_mic][3]; n_mic is read from mics' shape unless given."""
        import torch
        n_rir = int(geom.numel() // 10) if geom is not None else 0
        if n_mic is None:
            n_mic = int(mics.shape[-2]) if mics is not None and mics.dim() >= 2 else 0
        if self._check_sizes:
            check_rir_sizes(geom, rir_len, rir_out, tap_count_out, mics, int(n_mic))
        self._check(self._lib.aug_rir_mics_batch(
            self._h, n_rir, int(n_mic), _ptr(geom, torch.float32), _ptr(mics, torch.float32), int(rir_len),
            float(fs), float(c), _ptr(rir_out, torch.float32), _ptr(tap_count_out, torch.int32)))

    def aug_convolve_mix_batch(self, offsets, speech, noise, rir, rir_len: int, snr_db, mixed_out,
                               gains_out=None, n_noise: Optional[int] = None):
        import torch
        off = _host_i64(offsets)
        if n_noise is None:
            n_noise = 0 if noise is None else int(noise.shape[0])
        if self._check_sizes:
            check_convolve_mix_sizes(off, speech, int(n_noise), noise, rir, rir_len, snr_db, mixed_out, gains_out)
        self._check(self._lib.aug_convolve_mix_batch(
            self._h, len(off) - 1, off.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
            _ptr(speech, torch.float32), int(n_noise), _ptr(noise, torch.float32),
            _ptr(rir, torch.float32), int(rir_len), _ptr(snr_db, torch.float32),
            _ptr(mixed_out, torch.float32), _ptr(gains_out, torch.float32)))

    def aug_vtlp_mel_batch(self, offsets, wave, alpha, cfg, frame_offsets, feats_out):
        import torch
        off = _host_i64(offsets)
        foff = _host_i64(frame_offsets)
        c = cfg if isinstance(cfg, FrontendCfg) else FrontendCfg.of(cfg)
        if self._check_sizes:
            check_mel_sizes(off, foff, wave, alpha, feats_out, self._lib.aug_feature_dim(ctypes.byref(c)))
        self._check(self._lib.aug_vtlp_mel_batch(
            self._h, len(off) - 1, off.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
            _ptr(wave, torch.float32), _ptr(alpha, torch.float32), ctypes.byref(c),
            foff.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), _ptr(feats_out, torch.float32)))

    def aug_vtlp_mel_batch_static(self, offsets, wave, alpha, cfg, frame_offsets, feats_out):
        """aug_vtlp_mel_batch with its tables in the library's static device array: the call allocates nothing."""
        import torch
        off = _host_i64(offsets)
        foff = _host_i64(frame_offsets)
        c = cfg if isinstance(cfg, FrontendCfg) else FrontendCfg.of(cfg)
        if self._check_sizes:
            check_mel_sizes(off, foff, wave, alpha, feats_out, self._lib.aug_feature_dim(ctypes.byref(c)))
        self._check(self._lib.aug_vtlp_mel_batch_static(
            self._h, len(off) - 1, off.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
            _ptr(wave, torch.float32), _ptr(alpha, torch.float32), ctypes.byref(c),
            foff.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), _ptr(feats_out, torch.float32)))

    def aug_vtlp_resynth_batch(self, offsets, wave, alpha, wave_out, win: int = 800, hop: int = 400,
                               nfft: int = 2048):
        import torch
        off = _host_i64(offsets)
        c = VtlpCfg(int(win), int(hop), int(nfft))
        if self._check_sizes:
            check_resynth_sizes(off, wave, alpha, wave_out)
        self._check(self._lib.aug_vtlp_resynth_batch(
            self._h, len(off) - 1, off.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
            _ptr(wave, torch.float32), _ptr(alpha, torch.float32), ctypes.byref(c),
            _ptr(wave_out, torch.float32)))

    def aug_pipeline_batch(self, offsets, speech, noise, geom, rir_len: int, fs: float, c: float,
                           snr_db, alpha, cfg, frame_offsets, feats_out, rir_out=None,
                           mixed_out=None, gains_out=None, n_noise: Optional[int] = None):
        import torch
        off = _host_i64(offsets)
        foff = _host_i64(frame_offsets)
        fc = cfg if isinstance(cfg, FrontendCfg) else FrontendCfg.of(cfg)
        if n_noise is None:
            n_noise = 0 if noise is None else int(noise.shape[0])
        if self._check_sizes:
            check_pipeline_sizes(off, foff, speech, int(n_noise), noise, geom, rir_len, snr_db, alpha,
                                 self._lib.aug_feature_dim(ctypes.byref(fc)), feats_out, rir_out, mixed_out,
                                 gains_out)
        self._check(self._lib.aug_pipeline_batch(
            self._h, len(off) - 1, off.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
            _ptr(speech, torch.float32), int(n_noise), _ptr(noise, torch.float32),
            _ptr(geom, torch.float32), int(rir_len), float(fs), float(c),
            _ptr(snr_db, torch.float32), _ptr(alpha, torch.float32), ctypes.byref(fc),
            foff.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), _ptr(feats_out, torch.float32),
            _ptr(rir_out, torch.float32), _ptr(mixed_out, torch.float32),
            _ptr(gains_out, torch.float32)))

    # ---- operators on feature rows: matrices are [rows][columns] tensors, column slices of wider ones among them.  Their
    # shapes are checked whatever check_sizes says: the leading dimension comes from them. ----

    def _on_device(self, name, t):
        if t.get_device() != self.device:
            raise ValueError(f"{name} is on {t.device}, the context on device {self.device}")
        return t.data_ptr()

    # (the common case is settled in one expression: a step of a few streams takes the GPU less time than its arguments take here)

    def _matrix(self, name, t, n_rows, width, dtype):
        """The fields of aug_rows (None: no matrix)."""
        if t is None:
            return 0, 0
        if t.shape == (n_rows, width) and t.dtype is dtype and t.get_device() == self.device:
            down, across = t.stride()
            if across == 1 and down >= width:
                return t.data_ptr(), down
        ld = check_matrix(name, t, n_rows, width, dtype)
        return self._on_device(name, t), ld

    def _array(self, name, t, count, dtype=None):
        if t is None:
            return None
        if dtype is None:
            dtype = self._f32
        if t.numel() == count and t.dtype is dtype and t.is_contiguous() and t.get_device() == self.device:
            return t.data_ptr()
        check_array(name, t, count, dtype)
        return self._on_device(name, t)

    @staticmethod
    def _sequences(row_offsets, row_lengths):
        """n_seq, the rows that they reach, and the host arrays with their addresses."""
        off = _host_i64(row_offsets)
        lengths = None if row_lengths is None else _host_i64(row_lengths)
        n_rows = check_row_offsets(off, lengths)
        return len(off) - 1, n_rows, (off, lengths), off.ctypes.data, None if lengths is None else lengths.ctypes.data

    def aug_rms_norm_batch(self, x, weight=None, residual=None, eps: float = 1e-6, sum_out=None, y_out=None, q_out=None,
                           scale_out=None, rstd_out=None, q_block: int = 0):
        import torch
        n_rows, dim = _two_dimensions("x", x)
        m, arr, dtype = self._matrix, self._array, x.dtype
        q_type = dtype if q_out is None else q_out.dtype
        if q_type not in (torch.float8_e4m3fn, torch.uint8) and q_out is not None:
            raise TypeError(f"q_out is {q_type}, expected float8_e4m3fn (or uint8 for the same bits)")
        scales = n_rows * (-(-dim // q_block) if q_block > 0 else 1)
        self._check(self._lib.aug_rms_norm_batch(
            self._h, n_rows, ctypes.byref(NormCfg(_element_type(x), dim, eps, q_block)), ROWS(*m("x", x, n_rows, dim, dtype)),
            ROWS(*m("residual", residual, n_rows, dim, dtype)), arr("weight", weight, dim),
            ROWS(*m("sum_out", sum_out, n_rows, dim, dtype)), ROWS(*m("y_out", y_out, n_rows, dim, dtype)),
            ROWS(*m("q_out", q_out, n_rows, dim, q_type)), arr("scale_out", scale_out, scales), arr("rstd_out", rstd_out, n_rows)))

    def aug_rms_norm_backward_batch(self, x, rstd, dy, weight=None, dsum=None, dx_out=None, dweight_out=None):
        """x is the forward call's sum (its input where there was no residual)."""
        n_rows, dim = _two_dimensions("x", x)
        m, arr, dtype = self._matrix, self._array, x.dtype
        self._check(self._lib.aug_rms_norm_backward_batch(
            self._h, n_rows, ctypes.byref(NormCfg(_element_type(x), dim, 0.0, 0)), ROWS(*m("x", x, n_rows, dim, dtype)),
            arr("weight", weight, dim), arr("rstd", rstd, n_rows), ROWS(*m("dy", dy, n_rows, dim, dtype)),
            ROWS(*m("dsum", dsum, n_rows, dim, dtype)), ROWS(*m("dx_out", dx_out, n_rows, dim, dtype)),
            arr("dweight_out", dweight_out, dim)))

    def aug_short_conv_batch(self, row_offsets, x, weight, y_out, bias=None, activation: str = "silu", state_in=None,
                             state_out=None, row_lengths=None):
        n_seq, n_rows, _keep, off, lengths = self._sequences(row_offsets, row_lengths)
        dim, taps = _two_dimensions("weight", weight)
        m, arr, dtype, held = self._matrix, self._array, x.dtype, n_seq * (taps - 1) * dim
        self._check(self._lib.aug_short_conv_batch(
            self._h, n_seq, off, lengths, SHORT_CONV_CFG(_element_type(x), dim, taps, ACTIVATIONS[activation]),
            ROWS(*m("x", x, n_rows, dim, dtype)), arr("weight", weight, dim * taps), arr("bias", bias, dim),
            arr("state_in", state_in, held, dtype), arr("state_out", state_out, held, dtype), ROWS(*m("y_out", y_out, n_rows, dim, dtype))))

    def aug_short_conv_backward_batch(self, row_offsets, x, weight, dy, bias=None, activation: str = "silu", state_in=None,
                                      dx_out=None, dweight_out=None, dbias_out=None, row_lengths=None):
        n_seq, n_rows, _keep, off, lengths = self._sequences(row_offsets, row_lengths)
        dim, taps = _two_dimensions("weight", weight)
        m, arr, dtype = self._matrix, self._array, x.dtype
        self._check(self._lib.aug_short_conv_backward_batch(
            self._h, n_seq, off, lengths, SHORT_CONV_CFG(_element_type(x), dim, taps, ACTIVATIONS[activation]),
            ROWS(*m("x", x, n_rows, dim, dtype)), arr("weight", weight, dim * taps), arr("bias", bias, dim),
            arr("state_in", state_in, n_seq * (taps - 1) * dim, dtype), ROWS(*m("dy", dy, n_rows, dim, dtype)),
            ROWS(*m("dx_out", dx_out, n_rows, dim, dtype)), arr("dweight_out", dweight_out, dim * taps), arr("dbias_out", dbias_out, dim)))

    def aug_short_conv_step(self, x, weight, state_in, state_out, y_out, bias=None, activation: str = "silu"):
        n_seq = x.shape[0]
        dim, taps = _two_dimensions("weight", weight)
        m, arr, dtype, held = self._matrix, self._array, x.dtype, n_seq * (taps - 1) * dim
        self._check(self._lib.aug_short_conv_step(
            self._h, n_seq, SHORT_CONV_CFG(_element_type(x), dim, taps, ACTIVATIONS[activation]), ROWS(*m("x", x, n_seq, dim, dtype)),
            arr("weight", weight, dim * taps), arr("bias", bias, dim), arr("state_in", state_in, held, dtype),
            arr("state_out", state_out, held, dtype), ROWS(*m("y_out", y_out, n_seq, dim, dtype))))

    def _scan_in(self, n_rows, u, delta, a, b, c, skip, z, delta_bias, softplus, n_group):
        dim, n_state = _two_dimensions("a", a)
        m, arr, dtype, group = self._matrix, self._array, u.dtype, n_group * n_state
        return SCAN_CFG(_element_type(u), dim, n_state, n_group, bool(softplus)), SCAN_IN(
            *m("u", u, n_rows, dim, dtype), *m("delta", delta, n_rows, dim, dtype), *m("b", b, n_rows, group, dtype),
            *m("c", c, n_rows, group, dtype), *m("z", z, n_rows, dim, dtype), arr("a", a, dim * n_state),
            arr("skip", skip, dim) or 0, arr("delta_bias", delta_bias, dim) or 0)

    def aug_scan_batch(self, row_offsets, u, delta, a, b, c, y_out, skip=None, z=None, delta_bias=None, softplus: bool = True,
                       n_group: int = 1, state_in=None, state_out=None, row_lengths=None):
        n_seq, n_rows, _keep, off, lengths = self._sequences(row_offsets, row_lengths)
        cfg, ins = self._scan_in(n_rows, u, delta, a, b, c, skip, z, delta_bias, softplus, n_group)
        arr, held = self._array, n_seq * a.numel()
        self._check(self._lib.aug_scan_batch(self._h, n_seq, off, lengths, cfg, ins, arr("state_in", state_in, held),
                                             arr("state_out", state_out, held), ROWS(*self._matrix("y_out", y_out, n_rows, cfg[1], u.dtype))))

    def aug_scan_backward_batch(self, row_offsets, u, delta, a, b, c, dy, skip=None, z=None, delta_bias=None, softplus: bool = True,
                                n_group: int = 1, state_in=None, du_out=None, ddelta_out=None, da_out=None, db_out=None, dc_out=None,
                                dskip_out=None, ddelta_bias_out=None, dz_out=None, row_lengths=None):
        n_seq, n_rows, _keep, off, lengths = self._sequences(row_offsets, row_lengths)
        cfg, ins = self._scan_in(n_rows, u, delta, a, b, c, skip, z, delta_bias, softplus, n_group)
        m, arr, dtype, dim, group = self._matrix, self._array, u.dtype, cfg[1], cfg[2] * n_group
        out = SCAN_GRAD(
            *m("du_out", du_out, n_rows, dim, dtype), *m("ddelta_out", ddelta_out, n_rows, dim, dtype),
            *m("db_out", db_out, n_rows, group, dtype), *m("dc_out", dc_out, n_rows, group, dtype), *m("dz_out", dz_out, n_rows, dim, dtype),
            arr("da_out", da_out, a.numel()) or 0, arr("dskip_out", dskip_out, dim) or 0, arr("ddelta_bias_out", ddelta_bias_out, dim) or 0)
        self._check(self._lib.aug_scan_backward_batch(self._h, n_seq, off, lengths, cfg, ins, arr("state_in", state_in, n_seq * a.numel()),
                                                      ROWS(*m("dy", dy, n_rows, dim, dtype)), out))

    def aug_scan_step(self, u, delta, a, b, c, state_in, state_out, y_out, skip=None, z=None, delta_bias=None, softplus: bool = True,
                      n_group: int = 1):
        n_seq = u.shape[0]
        cfg, ins = self._scan_in(n_seq, u, delta, a, b, c, skip, z, delta_bias, softplus, n_group)
        arr, held = self._array, n_seq * a.numel()
        self._check(self._lib.aug_scan_step(self._h, n_seq, cfg, ins, arr("state_in", state_in, held), arr("state_out", state_out, held),
                                            ROWS(*self._matrix("y_out", y_out, n_seq, cfg[1], u.dtype))))
