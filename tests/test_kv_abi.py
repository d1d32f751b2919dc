"""CPU-side checks of the key-value cache ABI: header and binding agree, the header compiles alone, what needs no device is
right, and bad arguments are refused before CUDA is touched."""
import ctypes
import math
import os
import re
import subprocess

import pytest

from paper_2410_15240_b200 import fastrack, kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fastrack_kv.h")


def test_header_and_binding_agree():
    text = open(HEADER).read()
    names = sorted(set(re.findall(r"FASTRACK_API\s+[\w\s\*]+?\b(fastrack_\w+)\s*\(", text)))
    assert sorted(kv.EXPORTS) == names
    lib = ctypes.CDLL(fastrack.LIB_PATH)
    for name in names:
        assert hasattr(lib, name), name
    values = dict(re.findall(r"FASTRACK_((?:KV|ROTARY|FREQ)_\w+) = (\d)", text))
    for name, value in values.items():
        assert getattr(kv, name[3:] if name.startswith("KV_") else name) == int(value), name
    for struct, cls in (("config", kv.Config), ("batch", kv.Batch), ("rows", kv.Rows), ("eviction", kv.Eviction)):
        body = re.search(r"typedef struct \{([^}]*)\} fastrack_kv_%s;" % struct, text).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = [w.strip(" *") for line in body.split(";") for w in re.sub(r"^\s*(const )?\w+[ *]+", "", line.strip()).split(",") if line.strip()]
        assert fields == [f for f, _ in cls._fields_], struct


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("gcc", "-std=c11"), ("g++", "-std=c++11"), ("g++", "-std=c++17")])
def test_header_compiles_on_its_own(tmp_path, compiler, std):
    src = tmp_path / ("use.c" if compiler == "gcc" else "use.cpp")
    src.write_text('#include "fastrack_kv.h"\n#include "fastrack_kv.h"\nint use(const fastrack_kv* c) { return (int)fastrack_kv_page_bytes(c); }\n')
    subprocess.check_call([compiler, std, "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o",
                           str(tmp_path / "use.o")])


def test_null_handles():
    lib = fastrack._lib
    assert lib.fastrack_kv_create(None, None) == fastrack.ERR_ARG
    assert lib.fastrack_kv_page_bytes(None) == 0 and lib.fastrack_kv_tail_bytes(None) == 0
    assert lib.fastrack_kv_last_cuda_error(None) == 0 and lib.fastrack_kv_launch_count(None) == 0
    b, r, e = kv.Batch(), kv.Rows(), kv.Eviction()
    assert lib.fastrack_rotary(None, 1, 1, r, r, None, 0, None) == fastrack.ERR_ARG
    assert lib.fastrack_kv_append(None, b, r, r, None, None, None) == fastrack.ERR_ARG
    assert lib.fastrack_kv_read(None, b, r, r, None) == fastrack.ERR_ARG
    assert lib.fastrack_kv_attention_workspace(None, b, 0) == 0
    assert lib.fastrack_kv_attention(None, b, r, r, None, 0, None, None, 0, None, 0, None) == fastrack.ERR_ARG
    assert lib.fastrack_kv_evict(None, e, None) == fastrack.ERR_ARG
    lib.fastrack_kv_destroy(None)


BAD_CONFIGS = [dict(dtype=2), dict(format=-1), dict(q_heads=0), dict(q_heads=1025), dict(q_heads=9), dict(kv_heads=0), dict(head_dim=80), dict(block_tokens=48),
               dict(block_tokens=8), dict(rotary=3), dict(rotary=1), dict(rotary=1, frequencies=[1.0] * 7), dict(rotary=1, frequencies=[1.0] * 72),
               dict(rotary=2, frequencies=[1.0] * 7 + [math.inf]), dict(frequencies=[1.0] * 8), dict(rotary=1, frequencies=[1.0] * 8, rotary_gain=math.nan),
               dict(softmax_scale=math.inf), dict(softmax_scale=-0.1)]


@pytest.mark.parametrize("change", BAD_CONFIGS, ids=str)
def test_bad_configurations_are_refused(change):
    good = dict(dtype=kv.BF16, format=kv.INT8, q_heads=8, kv_heads=2, head_dim=128, block_tokens=64)
    with pytest.raises(fastrack.FastrackError) as e:
        kv.KvCache(**{**good, **change})
    assert e.value.code == fastrack.ERR_ARG


def test_no_cpu_fallback_without_a_device():
    import torch
    if torch.cuda.is_available():
        return
    with pytest.raises(fastrack.FastrackError) as e:
        kv.KvCache(kv.BF16, kv.INT8, 8, 2, 128, 64)
    assert e.value.code == fastrack.ERR_CUDA


# pow and the few products around it are within a few units of the last place of a double
CLOSE = dict(rel_tol=1e-14)


def test_frequencies():
    plain, gain = kv.rotary_frequencies(64, 10000.0)
    assert gain == 1.0 and len(plain) == 32
    assert all(math.isclose(f, 10000.0 ** (-2 * i / 64), **CLOSE) for i, f in enumerate(plain))
    linear, gain = kv.rotary_frequencies(64, 10000.0, kv.FREQ_LINEAR, 4.0)
    assert gain == 1.0 and all(math.isclose(f, p / 4, **CLOSE) for f, p in zip(linear, plain))
    based, gain = kv.rotary_frequencies(64, 10000.0, kv.FREQ_BASE, 4.0)
    assert gain == 1.0 and based[0] == 1.0 and math.isclose(based[-1], plain[-1] / 4, rel_tol=1e-12)
    assert all(a / 4 <= b * (1 + 1e-12) and b <= a for a, b in zip(plain, based))
    ramp, gain = kv.rotary_frequencies(64, 10000.0, kv.FREQ_RAMP, 4.0, 4096.0)
    assert math.isclose(gain, 0.1 * math.log(4) + 1, rel_tol=1e-6)
    for f, p in zip(ramp, plain):
        turns = 4096 * p / (2 * math.pi)
        if turns > 32:
            assert math.isclose(f, p, **CLOSE)
        elif turns < 1:
            assert math.isclose(f, p / 4, **CLOSE)
        else:
            assert p / 4 < f < p
    same, gain = kv.rotary_frequencies(64, 10000.0, kv.FREQ_RAMP, 1.0, 4096.0)
    assert gain == 1.0 and all(math.isclose(f, p, **CLOSE) for f, p in zip(same, plain))


@pytest.mark.parametrize("args", [(0,), (7,), (64, 1.0), (64, math.inf), (64, 1e4, 4), (64, 1e4, -1), (64, 1e4, 1, 0.5), (64, 1e4, 1, math.nan), (2, 1e4, 2, 2.0),
                                  (64, 1e4, 3, 2.0, 0.0), (64, 1e4, 3, 2.0, math.inf)])
def test_bad_frequencies_are_refused(args):
    with pytest.raises(fastrack.FastrackError):
        kv.rotary_frequencies(*args)
