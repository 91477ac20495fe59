"""The binding where the module of the token-step calls could not be built: every other call is there, those raise and say why."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_without_the_token_step_module_the_other_calls_work():
    code = """
import sys, types
sys.path.insert(0, %r)
sys.modules["paper_2601_08743_amd._py_step"] = None
from paper_2601_08743_amd import binding as B
assert B.tc_version() and B.tc_digest_bytes(B.make_config(1, 8, 2, 64, B.TC_F32, 10, 0, 16)) > 0
ctx = types.SimpleNamespace(_step=None)
calls = [lambda: B.Context.tc_step_tables(ctx, *[None] * 13), lambda: B.Context.tc_rope_append(ctx, 0, None, None, None, None, 1e4, None, None),
         lambda: B.Context.tc_digest_blocks(ctx, 0, 1, None, None), lambda: B.Context.tc_select_blocks(ctx, 0, *[None] * 5, 1, 1, 1, None, None),
         lambda: B.Context.tc_block_attn(ctx, 0, *[None] * 6, 0.1, None)]
for call in calls:
    try:
        call()
    except ImportError as e:
        assert "_py_step.so is not built" in str(e), e
    else:
        raise AssertionError("no error")
print("the others: ok")
""" % ROOT
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "the others: ok" in r.stdout, r.stdout + r.stderr
