"""Runs one case of operators.py three times through the library: what a profiler is given.

    python perf/run_case.py attend-decode-256
    python perf/run_case.py --sources      # the hash of the attention kernels' sources that the counter summaries carry
"""

import hashlib
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = ["lv_base.cuh", "lv_attend.cuh", "lv_chunk.cuh", "lv_decode.cuh", "lv_kv.cu", "lv_kv.h", "lv_kv_plan.cuh",
           "lv_kv_store.cuh", "lv_prompt.cuh", "lv_tc.cuh"]


def sources():
    """First 16 digits of the sha256 of the attention kernels' sources, one after another."""
    h = hashlib.sha256()
    for name in SOURCES:
        with open(os.path.join(ROOT, "paper_2608_08382_gb300", "csrc", name), "rb") as f:
            h.update(f.read())
    return h.hexdigest()[:16]


def run(name):
    sys.path.insert(0, ROOT)
    from perf import operators
    import torch
    operators.own = True
    state = operators.prepare(next(c for c in operators.listed() if c["name"] == name), 1)
    for _ in range(3):
        operators.run(state)
    torch.cuda.synchronize()


if __name__ == "__main__":
    if sys.argv[1] == "--sources":
        print(sources())
    else:
        run(sys.argv[1])
