"""Tables of thousands of requests, in a process that has made no larger call: what a launch may take of shared memory is
asked for by the call itself, not left over from an earlier one."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# Requests of one new token each; those whose length is a multiple of the block size lack a block.
SCRIPT = """
import sys
import numpy as np, torch
import serving_ref as R
from paper_2408_04323_gb300 import scoot as S

def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()

for n in map(int, sys.argv[1:]):
    cached, new, bs = np.arange(n) % 16, np.ones(n, int), 8
    table, free = np.stack([2 * np.arange(n), 2 * np.arange(n) + 1], 1), 2 * n + np.arange(n)
    table[cached <= 8, 1], table[cached == 0, 0] = -1, -1
    want = R.tables(cached, new, table, bs, 3 * n, free, n)
    t, out = i32(table), [torch.full((m,), -7, dtype=d, device="cuda") for m, d in
                          ((n + 1, torch.int32), (n, torch.int32), (n, torch.int64), (n, torch.int32), (2, torch.int32))]
    with S.Context(0) as ctx:
        S.scoot_kv_tables(ctx, i32(cached), i32(new), t, bs, 3 * n, i32(free), *out)
        ctx.check()
    for w, g in zip(want, (t, *out)):
        assert np.array_equal(w, g.cpu().numpy()), n
print("ok")
"""


@pytest.mark.parametrize("sizes", [(3007,), (3071,), (3006, 3040, 3073), (16384, 16385, 3050)], ids=str)
def test_tables_in_a_fresh_process(sizes):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2408_04323_gb300 as pkg
    pkg.build()
    path = os.pathsep.join([ROOT, os.path.join(ROOT, "tests"), os.environ.get("PYTHONPATH", "")])
    got = subprocess.run([sys.executable, "-c", SCRIPT, *map(str, sizes)], capture_output=True, text=True, timeout=300,
                         env={**os.environ, "PYTHONPATH": path}, cwd=ROOT)
    assert got.returncode == 0 and got.stdout.strip() == "ok", got.stderr[-2000:]
