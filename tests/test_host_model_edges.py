"""Edges of the model-side entry points that show without a GPU.  Calls that get
as far as a launch run in a child process that sees no device: there they end
in E_HIP, and a crash of the host code ends the child alone."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def child(code):
    """Status name that the call in `code` ends with ("OK" if none), in a process without a device."""
    text = ("import paper_2609_38767_amd as dt\nP = 1 << 20\ntry:\n" +
            "".join(f"    {line}\n" for line in code.splitlines()) +
            "    print('OK')\nexcept dt.DattriError as e:\n    print(e.status_name)\n")
    r = subprocess.run([sys.executable, "-c", text], cwd=ROOT, capture_output=True, text=True,
                       env=dict(os.environ, HIP_VISIBLE_DEVICES="-1"))
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])
    return r.stdout.split()[-1]


@pytest.mark.parametrize("vocab", [1, 262143, 262144, (1 << 31) - 1])
def test_embedding_grad_without_tokens(vocab):
    """No tokens and a table of any size: on to the launch that zeroes the table, through no division by zero work."""
    ws = "dt.dattri_embedding_grad_workspace_bytes(0, %d, 4)" % vocab
    call = "dt.dattri_embedding_grad(None, 0, 1, None, 8, 0, 1.0, %d, 4, P, 0, %d, 2 * P, %s, 0)"
    assert child(call % (vocab, 0, ws)) == "E_HIP"
    assert child(call % (vocab, 1, ws)) == "OK"  # nothing is added: no launch
