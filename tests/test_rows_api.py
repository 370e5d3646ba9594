"""The operators on feature rows without a GPU: what the C ABI refuses and how it recovers from running out of memory (its API layer on a
host runtime), and what the binding refuses before the library sees it."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_1912_11040_amd import binding as B
from paper_1912_11040_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
ROCM_INCLUDE = "/opt/rocm/include"


@pytest.mark.skipif(not shutil.which("g++") or not os.path.isdir(ROCM_INCLUDE), reason="needs g++ and the HIP headers")
def test_api_layer(tmp_path):
    exe = str(tmp_path / "rows_api")
    csrc = os.path.join(HERE, "..", "paper_1912_11040_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-D__HIP_PLATFORM_AMD__", "-D__align__(n)=__attribute__((aligned(n)))", "-DHIP_SYMBOL(s)=s",
                    "-I" + ROCM_INCLUDE, "-I" + os.path.join(HERE, "..", "include"), "-I" + csrc, os.path.join(HERE, "host", "rows_api.cpp"),
                    "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    print(r.stdout[-3000:])
    assert r.returncode == 0


def _fields(name):
    hdr = open(os.path.join(HERE, "..", "include", "aug.h")).read()
    body = re.sub(r"/\*.*?\*/", "", hdr[:hdr.index("} %s;" % name)].rsplit("typedef struct %s {" % name, 1)[1], flags=re.S)
    return [f.strip(" *") for _, names in re.findall(r"^\s*(?:const\s+)?(\w+)\s*\**\s*([\w\s,*]+);", body, flags=re.M) for f in names.split(",")]


def test_structs_match_the_header():
    assert _fields("aug_rows") == ["data", "ld"] and ctypes.sizeof(B.ROWS) == 16
    assert _fields("aug_norm_cfg") == [f[0] for f in B.NormCfg._fields_] and ctypes.sizeof(B.NormCfg) == 16
    assert _fields("aug_short_conv_cfg") == ["dtype", "dim", "taps", "silu"] and ctypes.sizeof(B.SHORT_CONV_CFG) == 16
    assert _fields("aug_scan_cfg") == ["dtype", "dim", "n_state", "n_group", "softplus"] and ctypes.sizeof(B.SCAN_CFG) == 20
    assert _fields("aug_scan_in") == ["u", "delta", "b", "c", "z", "a", "skip", "delta_bias"] and ctypes.sizeof(B.SCAN_IN) == 5 * 16 + 3 * 8
    assert _fields("aug_scan_grad") == ["du", "ddelta", "db", "dc", "dz", "da", "dskip", "ddelta_bias"] and ctypes.sizeof(B.SCAN_GRAD) == 5 * 16 + 3 * 8


def test_stages_match_the_header():
    hdr = open(os.path.join(HERE, "..", "include", "aug.h")).read()
    names = re.findall(r"^    AUG_STAGE_(\w+)", hdr, flags=re.M)
    assert [n.lower() for n in names] == list(B.STAGES)


@pytest.fixture(scope="module")
def host():
    """A binding object whose tensors live on the host and whose context is null: a call that passes the binding's checks is refused by the
    library before anything else happens."""
    if not os.path.exists(B.LIB_PATH):
        build.build()
    a = B.Augmenter.__new__(B.Augmenter)
    a._lib, a._check_sizes, a._f32, a.device, a._h = B.load_library(), True, torch.float32, -1, None
    return a


OFF = np.array([0, 5, 5, 12], np.int64)
BF = torch.bfloat16


def m(rows, width, dtype=BF):
    return torch.zeros(rows, width, dtype=dtype)


def reaches_the_library(call):
    with pytest.raises(B.AugError, match="context is null"):
        call()


def norm_args():
    return dict(x=m(6, 40), weight=torch.zeros(40), residual=m(6, 40), sum_out=m(6, 40), y_out=m(6, 40),
                q_out=m(6, 40, torch.float8_e4m3fn), scale_out=torch.zeros(6, 3), rstd_out=torch.zeros(6), q_block=16)


def norm_back_args():
    return dict(x=m(6, 40), rstd=torch.zeros(6), dy=m(6, 40), weight=torch.zeros(40), dsum=m(6, 40), dx_out=m(6, 40), dweight_out=torch.zeros(40))


def conv_args():
    return dict(row_offsets=OFF, x=m(12, 80)[:, 40:], weight=torch.zeros(40, 4), y_out=m(14, 40), bias=torch.zeros(40),
                state_in=torch.zeros(3, 3, 40, dtype=BF), state_out=torch.zeros(3, 3, 40, dtype=BF))


def conv_back_args():
    return dict(row_offsets=OFF, x=m(12, 40), weight=torch.zeros(40, 4), dy=m(12, 40), bias=torch.zeros(40), dx_out=m(12, 40),
                state_in=torch.zeros(3, 3, 40, dtype=BF), dweight_out=torch.zeros(40, 4), dbias_out=torch.zeros(40))


def conv_step_args():
    return dict(x=m(3, 40), weight=torch.zeros(40, 4), state_in=torch.zeros(3, 3, 40, dtype=BF), state_out=torch.zeros(3, 3, 40, dtype=BF), y_out=m(3, 40))


def scan_args(rows=12):
    bc = m(rows, 96)
    return dict(u=m(rows, 40), delta=m(rows, 40), a=torch.zeros(40, 16), b=bc[:, 32:64], c=bc[:, 64:], skip=torch.zeros(40), z=m(rows, 40),
                delta_bias=torch.zeros(40), n_group=2)


def scan_batch_args():
    return dict(row_offsets=OFF, y_out=m(12, 40), state_in=torch.zeros(3, 40, 16), state_out=torch.zeros(3, 40, 16), **scan_args())


def scan_back_args():
    return dict(row_offsets=OFF, dy=m(12, 40), state_in=torch.zeros(3, 40, 16), du_out=m(12, 40), ddelta_out=m(12, 40), db_out=m(12, 32),
                dc_out=m(12, 32), dz_out=m(12, 40), da_out=torch.zeros(40, 16), dskip_out=torch.zeros(40), ddelta_bias_out=torch.zeros(40), **scan_args())


def scan_step_args():
    return dict(y_out=m(3, 40), state_in=torch.zeros(3, 40, 16), state_out=torch.zeros(3, 40, 16), **scan_args(3))


CALLS = {"aug_rms_norm_batch": norm_args, "aug_rms_norm_backward_batch": norm_back_args, "aug_short_conv_batch": conv_args,
         "aug_short_conv_backward_batch": conv_back_args, "aug_short_conv_step": conv_step_args, "aug_scan_batch": scan_batch_args,
         "aug_scan_backward_batch": scan_back_args, "aug_scan_step": scan_step_args}


@pytest.mark.parametrize("name", CALLS)
def test_well_formed_calls_reach_the_library(host, name):
    reaches_the_library(lambda: getattr(host, name)(**CALLS[name]()))
    optional = {"residual", "bias", "z", "skip", "delta_bias", "dsum", "weight" if "norm" in name else "", "dz_out"}
    reaches_the_library(lambda: getattr(host, name)(**{k: None if k in optional else v for k, v in CALLS[name]().items()}))


@pytest.mark.parametrize("name", CALLS)
def test_every_tensor_is_checked(host, name):
    """A column or element short, a row short, another type, columns apart: each tensor of each call."""
    for k, v in CALLS[name]().items():
        if not isinstance(v, torch.Tensor):
            continue
        first = k in ("x", "u")                           # the others are compared with its type, and single rows with its number
        wrong = [v[:, :-1] if v.dim() > 1 else v[:-1]]
        if not (first and ("step" in name or "norm" in name)):
            wrong.append(v[:-1])
        if k == "y_out" and name == "aug_short_conv_batch":
            wrong[1] = v[:11]                             # (it has rows to spare)
        if not first:
            wrong.append(v.to(torch.float64))
        if v.dim() == 2 and v.shape[1] > 1:
            wrong.append(v.t().contiguous().t())          # columns that are not next to each other
        for w in wrong:
            with pytest.raises((ValueError, TypeError)):
                getattr(host, name)(**{**CALLS[name](), k: w})


def test_types_and_sequences_are_checked(host):
    with pytest.raises(TypeError):
        host.aug_rms_norm_batch(m(2, 8, torch.float64), None, y_out=m(2, 8, torch.float64))
    with pytest.raises(KeyError):
        host.aug_short_conv_step(**conv_step_args(), activation="relu")
    for lengths in ([1, 2], [[1, 2, 3]]):
        with pytest.raises(ValueError, match="row_lengths"):
            host.aug_scan_batch(**scan_batch_args(), row_lengths=lengths)
    with pytest.raises(ValueError, match="12 rows"):
        host.aug_scan_batch(**{**scan_batch_args(), "y_out": m(11, 40)})
    reaches_the_library(lambda: host.aug_scan_batch(**{**scan_batch_args(), "y_out": m(11, 40)[:11], "u": m(11, 40), "delta": m(11, 40), "z": m(11, 40),
                                                       "b": m(11, 32), "c": m(11, 32)}, row_lengths=[5, 0, 6]))


def test_overlapping_rows_are_refused(host):
    x = torch.as_strided(torch.zeros(200, dtype=BF), (6, 40), (20, 1))
    with pytest.raises(ValueError, match="overlap"):
        host.aug_rms_norm_batch(x, None, y_out=m(6, 40))
