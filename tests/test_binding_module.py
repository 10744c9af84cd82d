"""The C++ module that marshals the e4m3 and expert-layer calls: the other calls do without it, and it is built again
for another torch."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2009_06488_b200 import build
    build.build()


def python(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)


def test_other_calls_do_not_need_the_module():
    r = python("import sys\n"
               "sys.modules['paper_2009_06488_b200._q4_torch'] = None          # as if it had not been built\n"
               "from paper_2009_06488_b200 import binding as q4\n"
               "assert q4.q4_gemm_workspace_bytes(4096, 4096, 4096) >= 0 and q4.q4_expert_sort_rows(100, 8, 16) == 208\n"
               "try:\n"
               "    q4.q4_expert_combine(None, None, None, None)\n"
               "except ImportError as e:\n"
               "    print('needs', e)\n")
    assert r.returncode == 0, r.stderr
    assert r.stdout.startswith("needs") and "python -m paper_2009_06488_b200.build" in r.stdout


def test_a_module_built_for_another_torch_is_refused():
    r = python("import sys, types\n"
               "m = types.ModuleType('paper_2009_06488_b200._q4_torch')\n"
               "m.built_for = '1.0'\n"
               "import paper_2009_06488_b200 as p\n"
               "sys.modules[m.__name__] = p._q4_torch = m\n"
               "from paper_2009_06488_b200 import binding as q4\n"
               "try:\n"
               "    q4.q4_expert_combine(None, None, None, None)\n"
               "except ImportError as e:\n"
               "    print('refused', e)\n")
    assert r.returncode == 0, r.stderr
    assert r.stdout.startswith("refused") and "torch 1.0" in r.stdout


def test_the_module_is_loaded_once():
    from paper_2009_06488_b200 import binding as q4
    with pytest.raises(TypeError):
        q4.q4_expert_combine(None, None, None, None)
    assert q4._t is q4._marshalling()


def test_another_torch_has_it_built_again(monkeypatch, tmp_path):
    from paper_2009_06488_b200 import build
    calls = []
    monkeypatch.setattr(build, "build_torch", lambda: calls.append(1))
    build.build()
    assert not calls
    monkeypatch.setattr(build, "TORCH_STAMP", str(tmp_path / "built_for"))
    (tmp_path / "built_for").write_text("1.0 cpython-312")
    build.build()
    assert len(calls) == 1
    (tmp_path / "built_for").unlink()
    build.build()
    assert len(calls) == 2
