"""CPU-side checks of the latent cache ABI: header and binding agree, the header compiles alone, and bad arguments are refused before CUDA is
touched."""
import ctypes
import math
import os
import re
import subprocess

import pytest

from paper_2410_15240_b200 import fastrack, kv, latent

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fastrack_latent.h")


def test_header_and_binding_agree():
    text = open(HEADER).read()
    names = sorted(set(re.findall(r"FASTRACK_API\s+[\w\s\*]+?\b(fastrack_\w+)\s*\(", text)))
    assert sorted(latent.EXPORTS) == names
    lib = ctypes.CDLL(fastrack.LIB_PATH)
    for name in names:
        assert hasattr(lib, name), name
    assert latent.TREE_MOST == int(re.search(r"FASTRACK_LATENT_TREE_MOST = (\d+)", text).group(1))
    for struct, cls in (("config", latent.Config), ("batch", latent.Batch), ("acceptance", latent.Acceptance)):
        body = re.search(r"typedef struct \{([^}]*)\} fastrack_latent_%s;" % struct, text).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = [w.strip(" *") for line in body.split(";") for w in re.sub(r"^\s*(const )?\w+[ *]+", "", line.strip()).split(",") if line.strip()]
        assert fields == [f for f, _ in cls._fields_], struct


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("gcc", "-std=c11"), ("g++", "-std=c++11"), ("g++", "-std=c++17")])
def test_header_compiles_on_its_own(tmp_path, compiler, std):
    src = tmp_path / ("use.c" if compiler == "gcc" else "use.cpp")
    src.write_text('#include "fastrack_latent.h"\n#include "fastrack_latent.h"\nint use(const fastrack_latent* c) { return (int)fastrack_latent_page_bytes(c); }\n')
    subprocess.check_call([compiler, std, "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o",
                           str(tmp_path / "use.o")])


def test_null_handles():
    lib = fastrack._lib
    assert lib.fastrack_latent_create(None, None) == fastrack.ERR_ARG
    assert lib.fastrack_latent_page_bytes(None) == 0 and lib.fastrack_latent_last_cuda_error(None) == 0 and lib.fastrack_latent_launch_count(None) == 0
    b, r, a = latent.Batch(), kv.Rows(), latent.Acceptance()
    assert lib.fastrack_latent_append(None, b, r, r, None, None, None, None) == fastrack.ERR_ARG
    assert lib.fastrack_latent_attention_workspace(None, b) == 0 and lib.fastrack_latent_prompt_workspace(None, b) == 0
    assert lib.fastrack_latent_attention(None, b, r, r, r, None, None, None, 0, None) == fastrack.ERR_ARG
    assert lib.fastrack_latent_expand(None, b, None, r, r, None, 0, None) == fastrack.ERR_ARG
    assert lib.fastrack_latent_prompt(None, b, r, r, r, r, None, 0, r, None, None, 0, None) == fastrack.ERR_ARG
    assert lib.fastrack_latent_accept(None, b, a, None) == fastrack.ERR_ARG
    lib.fastrack_latent_destroy(None)


BAD_CONFIGS = [dict(dtype=2), dict(dtype=-1), dict(heads=0), dict(heads=1025), dict(latent_dim=64), dict(latent_dim=192), dict(latent_dim=640), dict(rope_dim=0),
               dict(rope_dim=48), dict(rope_dim=128), dict(key_dim=96), dict(key_dim=0), dict(value_dim=256), dict(block_tokens=8), dict(block_tokens=48),
               dict(block_tokens=256), dict(rotary=3), dict(rotary=-1), dict(rotary=1), dict(frequencies=[1.0] * 32),
               dict(rotary=2, frequencies=[1.0] * 31 + [math.inf]), dict(rotary=1, frequencies=[1.0] * 32, rotary_gain=math.nan), dict(norm_eps=-1.0),
               dict(norm_eps=math.nan), dict(softmax_scale=math.inf), dict(softmax_scale=-0.1)]


@pytest.mark.parametrize("change", BAD_CONFIGS, ids=str)
def test_bad_configurations_are_refused(change):
    good = dict(dtype=kv.BF16, heads=8, latent_dim=512, rope_dim=64, key_dim=128, value_dim=128, block_tokens=64)
    with pytest.raises(fastrack.FastrackError) as e:
        latent.LatentCache(**{**good, **change})
    assert e.value.code == fastrack.ERR_ARG


def test_the_wrong_number_of_frequencies_is_refused():
    with pytest.raises(ValueError):
        latent.LatentCache(kv.BF16, 8, 512, 64, 128, 128, 64, rotary=kv.ROTARY_HALF, frequencies=[1.0] * 31)


def test_no_cpu_fallback_without_a_device():
    import torch
    if torch.cuda.is_available():
        return
    with pytest.raises(fastrack.FastrackError) as e:
        latent.LatentCache(kv.BF16, 8, 512, 64, 128, 128, 64)
    assert e.value.code == fastrack.ERR_CUDA
