"""B200-native GPU side of Fastrack's CPU<->GPU secure channel (arXiv 2410.15240).

``paper_2410_15240_b200.fastrack`` and ``.kv`` are the ctypes bindings of the C-ABI CUDA library (they raise at
import time if the library has not been built); ``paper_2410_15240_b200.synth`` holds the seeded
synthetic input generators.  Nothing here falls back to a CPU implementation.
"""
__all__ = ["fastrack", "kv", "synth"]
