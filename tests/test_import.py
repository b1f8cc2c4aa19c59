"""The package without torch: its host calls need none."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _python(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return r.stdout


def test_host_calls_without_torch():
    _python("import sys; sys.modules['torch'] = None; import paper_2607_19368_amd as P; "
            "W, psi, R = P.slh_gen_params(0, 24, 256, 1, 1); assert W.shape == (24, 256); P.load()")


def test_attention_is_loaded_when_it_is_asked_for():
    _python("import sys, paper_2607_19368_amd as P; assert 'torch' not in sys.modules; P.slh_attend; assert 'torch' in sys.modules; "
            "from paper_2607_19368_amd import slh_kv_append; assert P.attention.slh_kv_append is slh_kv_append")
    _python("from paper_2607_19368_amd import *; slh_attend_paged, slh_merge, slh_rope_table, load, slh")
    _python("import paper_2607_19368_amd as P; assert not hasattr(P, 'slh_nothing') and 'slh_attend' in dir(P)")
