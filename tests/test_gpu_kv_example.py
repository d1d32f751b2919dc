"""The cache, its eviction and the sealed transfers together, as examples/sealed_cache.py uses them."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_sealed_cache():
    spec = importlib.util.spec_from_file_location("sealed_cache", os.path.join(ROOT, "examples", "sealed_cache.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    r = module.main(verbose=False)
    blocks = sum((module.PROMPT - 97 * i + module.STEPS) // module.BLOCK - module.BUDGET for i in range(module.SEQS))
    assert r["evicted"] == blocks
    assert r["refused"] == [blocks // 2] and r["accepted"]
    assert r["same"], "pages that were sealed and brought back answer differently"
    assert 0.0 < r["kept_weight"] < 1.0
