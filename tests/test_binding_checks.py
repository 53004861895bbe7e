"""The binding's checks of shapes and types guard raw pointers: they hold under python -O."""
import ast
import os
import subprocess
import sys

from paper_2607_20652_amd import binding as dpb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import torch
from paper_2607_20652_amd import binding as dpb
assert False, "not under -O"
q, k, i = torch.zeros(1, 2, 4, 64), torch.zeros(1, 3, 2, 64), torch.zeros(2, dtype=torch.int64)
m, u8 = torch.zeros(512), torch.zeros(512).to(torch.float8_e4m3fn)
one = [torch.zeros(3)]
calls = [
    lambda: dpb.attention(q, k, k[..., :32]),
    lambda: dpb.attention(q, k, k.double()),
    lambda: dpb.attention(q, k[0], k[0]),
    lambda: dpb.attention(q, k, k, q_lens=i),
    lambda: dpb.attention(q, k, k, out=q[:, :1]),
    lambda: dpb.attention(q, k, k, lse=q),
    lambda: dpb.attention_bwd(q[:, :1], q, k, k, q, q[..., 0]),
    lambda: dpb.attention_bwd(q, q, k, k, q, q[..., 0], dk=q),
    lambda: dpb.adamw_step(one, [], m, m, step=1, lr=1.0),
    lambda: dpb.adamw_step(one, [torch.zeros(2)], m, m, step=1, lr=1.0),
]
for at, call in enumerate(calls):
    try:
        call()
    except AssertionError:
        continue
    except Exception as e:
        raise SystemExit(f"call {at}: {type(e).__name__} {e}")
    raise SystemExit(f"call {at} went through")
"""


def test_checks_hold_under_O():
    got = subprocess.run([sys.executable, "-O", "-c", CALLS], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert got.returncode == 0, got.stdout + got.stderr


def test_no_check_is_an_assert_statement():
    tree = ast.parse(open(dpb.__file__).read())
    assert not [n.lineno for n in ast.walk(tree) if isinstance(n, ast.Assert)]
