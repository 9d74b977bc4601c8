"""Calls of the device-side step that its other tests do not make: row counts around the kernels' limits."""
import os
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)                                            # as a script too
from test_gpu_device_step import slot_case

pytestmark = pytest.mark.gpu


def slots_steps(rows, in_place):
    """Three steps of a batch with room for 9000 tokens against the model."""
    rng = np.random.default_rng(rows)
    c = slot_case(rng, rows, 16, 40, 6, rows * 6, 9000, in_place=in_place)
    for _ in range(3):
        new = rng.integers(0, 4, rows)
        new[rng.random(rows) < 0.1] = -1
        c.step(new.tolist())


@pytest.mark.parametrize("rows,in_place", [(3024, False), (3025, False), (3050, True), (3071, False), (4096, False), (4097, True)])
def test_slots_as_a_process_first_call(rows, in_place):
    """The rows' scanned counts take 16 bytes of shared memory each: around what a kernel has without asking for more, the
    call may not depend on what an earlier call of the process has asked for."""
    p = subprocess.run([sys.executable, os.path.abspath(__file__), str(rows), str(int(in_place))], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout[-2000:] + p.stderr[-2000:]


if __name__ == "__main__":
    slots_steps(int(sys.argv[1]), bool(int(sys.argv[2])))
