"""Runs one case of operators.py or more_operators.py three times through the library: what a profiler is given.

    python perf/run_case.py attend-decode-256
    python perf/run_case.py --sources        # the hash of the attention kernels' sources that the counter summaries carry
    python perf/run_case.py --layer-sources  # that of the sources of a step's work for each token
"""

import hashlib
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = ["lv_base.cuh", "lv_attend.cuh", "lv_chunk.cuh", "lv_decode.cuh", "lv_kv.cu", "lv_kv.h", "lv_kv_plan.cuh",
           "lv_kv_store.cuh", "lv_prompt.cuh", "lv_tc.cuh"]
LAYER_SOURCES = ["lv_base.cuh", "lv_attend.cuh", "lv_cut.h", "lv_kv_store.cuh", "lv_layer.cu", "lv_linear.cuh",
                 "lv_logprobs.cuh", "lv_rotate.cuh", "lv_tc.cuh"]


def sources(names):
    """First 16 digits of the sha256 of these sources, one after another."""
    h = hashlib.sha256()
    for name in names:
        with open(os.path.join(ROOT, "paper_2608_08382_gb300", "csrc", name), "rb") as f:
            h.update(f.read())
    return h.hexdigest()[:16]


def run(name):
    sys.path.insert(0, ROOT)
    from perf import more_operators, operators
    import torch
    module, case = next((m, c) for m in (operators, more_operators) for c in m.listed() if c["name"] == name)
    module.own = True
    state = module.prepare(case, 1)
    for _ in range(3):
        module.run(state)
    torch.cuda.synchronize()


if __name__ == "__main__":
    if sys.argv[1] in ("--sources", "--layer-sources"):
        print(sources(SOURCES if sys.argv[1] == "--sources" else LAYER_SOURCES))
    else:
        run(sys.argv[1])
