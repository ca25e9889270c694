"""The binding's native marshalling builds, and works, where torch's headers have no DLPack exchange functions: every
tensor is read by its attributes then (CPU only)."""
import importlib.machinery
import importlib.util
import os
import subprocess
import sysconfig

import pytest
import torch

from paper_2602_00125_amd import binding as b
from paper_2602_00125_amd import build

OLD_HEADER = """#pragma once
#define DLPACK_MAJOR_VERSION 1
#define DLPACK_MINOR_VERSION 0
typedef struct { void* data; } DLTensor;
"""


@pytest.mark.parametrize("header", [None, OLD_HEADER, "typedef struct { void* data; } DLTensor;\n"], ids=["none", "old", "unnumbered"])
def test_builds_without_the_exchange_functions(header, tmp_path):
    include = tmp_path / "include"
    (include / "ATen").mkdir(parents=True)
    if header is not None:
        (include / "ATen" / "dlpack.h").write_text(header)
    out = str(tmp_path / ("_marshal" + sysconfig.get_config_var("EXT_SUFFIX")))
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-fPIC", "-shared", "-Wall", "-Werror", "-I", str(include), "-I",
           sysconfig.get_paths()["include"], os.path.join(build.CSRC, "pymarshal.cpp"), "-o", out, "-ldl"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    loader = importlib.machinery.ExtensionFileLoader("_marshal", out)
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("_marshal", loader))
    loader.exec_module(m)
    m.init(*b._INIT)
    with pytest.raises(ValueError, match="device tensors"):
        m.dropout_fwd(torch.zeros(2, 2), None, 0.0, 0, 0, torch.zeros(2, 2), 0)
    assert m.linear_fwd(None, None, None, None, 0) == 1  # MT_ERR_NULL: it reached the library

    class Made:
        is_cuda, dtype, shape = True, torch.float32, (2, 4)
        stride, data_ptr = (lambda self: (4, 1)), (lambda self: 4096)

    assert m.layer_norm_fwd(Made(), None, None, 1e-5, Made(), 0) == 6  # MT_ERR_ALIAS: both descriptors were read
