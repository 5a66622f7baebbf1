"""Host memory that runs out inside a call is a status, not an exception through the
C interface (which would end the process). Each case runs in a process of its own
that limits its address space."""

import os
import subprocess
import sys

import pytest

import paper_2512_04013_amd as aug

pytestmark = pytest.mark.skipif(not os.path.exists(aug.LIB_PATH), reason="libaug.so not built")

HEAD = """
import resource, sys
import numpy as np
import paper_2512_04013_amd as aug

aug.lib()

def limit(megabytes):
    with open("/proc/self/statm") as f:
        now = int(f.read().split()[0]) * resource.getpagesize()
    resource.setrlimit(resource.RLIMIT_AS, (now + (megabytes << 20),) * 2)

def refused(call):
    try:
        call()
    except aug.AugError as e:
        assert e.status == aug.AUG_ERR_NO_SPACE and "memory" in str(e), e
        print("refused", flush=True)
    else:
        raise SystemExit("not refused")
"""

# the planner looks for shared blocks in a table over a pool of 2^31 - 1 blocks: 268 MB of bits
PLAN = HEAD + """
s = aug.make_shape(8, 8, 128, "bf16", "bf16", "bf16", 0.1)
ids = np.arange(3125, dtype=np.int32)
span = dict(row_first=[0], row_end=[49990]) if sys.argv[1] == "masked" else {}
aug.aug_attn_plan(s, [0, 1], [50000], [0, 3125], 4000, ids, **span)
limit(64)
refused(lambda: aug.aug_attn_plan(s, [0, 1], [50000], [0, 3125], 2 ** 31 - 1, ids, **span))
if sys.argv[1] == "plain":
    refused(lambda: aug.aug_attn_workspace_size(s, [0, 1], [50000], [0, 3125], 2 ** 31 - 1, ids))
info, _ = aug.aug_attn_plan(s, [0, 1], [50000], [0, 3125], 4000, ids, **span)      # and goes on
assert info.num_items > 0
"""

# the former keeps a priority for each of its 5 million requests: 40 MB
FORM = HEAD + """
r = np.zeros(5_000_000, aug.REQUEST_DTYPE)
r["state"] = aug.AUG_PAUSED
p = aug.former_params()
aug.aug_form_batch(r, 10, 0.0, p)
few = r[:10].copy()
limit(8)
refused(lambda: aug.aug_form_batch(r, 10, 0.0, p))
assert len(aug.aug_form_batch(few, 10, 0.0, p)["ids"]) == 0
"""


@pytest.mark.parametrize("code,arg,times", [(PLAN, "plain", 2), (PLAN, "masked", 1), (FORM, "", 1)], ids=["plan", "masked", "former"])
def test_exhausted_memory_is_reported(code, arg, times):
    env = dict(os.environ, OPENBLAS_NUM_THREADS="1", OMP_NUM_THREADS="1")
    r = subprocess.run([sys.executable, "-c", code, arg], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr[-2000:])
    assert r.stdout.split() == ["refused"] * times
