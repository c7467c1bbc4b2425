"""What importing and building the package needs: networks need the library
alone; the operators their binding too, and they say so."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytest.importorskip("paper_2609_16742_amd.ctc")


def _python(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, text=True,
                       capture_output=True)
    assert r.returncode == 0, r.stderr
    return r.stdout


def test_networks_do_without_the_operators_binding():
    out = _python(
        "import sys\n"
        "sys.modules['paper_2609_16742_amd._binding'] = None\n"
        "import paper_2609_16742_amd as P\n"
        "P.CtcNet, P.ctc.ctc_abi_version()\n"
        "for f in (lambda: P.ops, lambda: __import__('paper_2609_16742_amd.ops')):\n"
        "    try:\n"
        "        f()\n"
        "    except ImportError as e:\n"
        "        print(e)\n")
    assert out.count("binding is not built") == 2 and "build" in out


def test_operators_are_found_by_every_spelling():
    _python("import paper_2609_16742_amd as P; P.ops.group_norm")
    _python("from paper_2609_16742_amd import ops; ops.group_norm")
    _python("import paper_2609_16742_amd.ops as ops; ops.group_norm")
    _python("import paper_2609_16742_amd as P\n"
            "try:\n    P.nothing\nexcept AttributeError as e:\n    assert 'nothing' in str(e)")


@pytest.mark.parametrize("binding", [False, True])
def test_the_library_builds_alone(monkeypatch, binding):
    from paper_2609_16742_amd import build as b
    ran = []
    monkeypatch.setattr(b, "_run", lambda cmd, verbose: ran.append(cmd))
    monkeypatch.setattr(b.os, "replace", lambda src, dst: None)
    b.build(binding=binding)
    assert len(ran) == 1 + binding
    assert ("--offload-arch=gfx950" in ran[0]) and (ran[0][0] != "g++")
