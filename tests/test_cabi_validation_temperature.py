"""The row operators' temperature: its reciprocal has to be a float, so what is below the smallest normal float is refused.  Checked like
test_cabi_validation_mx4.py, in a child process without a device: a call that is accepted reaches CUDA and reports QUAFF_ERR_CUDA."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r'''
import json, sys
from paper_2505_14742_b200 import binding as Q
L = Q.lib()
P = lambda i: 0x7F0000000000 + i * 0x100000
tau = float(sys.argv[1])
print(json.dumps([L.quaff_topk_logits(P(1), 0, 1000, 64, 1000, 20, tau, P(2), P(3), None, None),
                  L.quaff_distill_topk(P(1), 0, 1000, 64, 1000, P(2), P(3), 20, None, tau, None, P(4), P(5), 1000, None)]))
'''


@pytest.mark.parametrize("tau,want", [(1e-45, 1), (2.0 ** -127, 1), (2.0 ** -126, 5), (1e-3, 5), (3e38, 5)])
def test_temperatures(tau, want):
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="", PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    r = subprocess.run([sys.executable, "-c", CHILD, repr(tau)], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-2000:])
    assert json.loads(r.stdout.strip().splitlines()[-1]) == [want, want]
