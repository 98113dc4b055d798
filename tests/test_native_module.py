"""Where the module of the 8-bit operators' calls cannot be loaded, everything else works and a call of them says what to do (no GPU)."""
import os
import subprocess
import sys

from paper_2506_16235_b200 import build as nsml_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT = """
import sys
sys.modules["paper_2506_16235_b200._native"] = None  # as if it had not been built
import torch
import paper_2506_16235_b200 as nsml
from paper_2506_16235_b200 import dp
ctrl = nsml.Controller()
assert 0 < ctrl.select_ratio(0.0, 0.0, 1e6) <= 1
assert nsml.nsml_payload_bytes(1 << 20, 0.01, 8) > 0 and nsml.alloc_bytes(100, "cpu").numel() == 256
for call in (lambda: nsml.nsml_q8_pack(torch.zeros(2, 16)), lambda: nsml.nsml_q8_rms_norm(torch.zeros(2, 16), torch.ones(16)),
             lambda: dp.NormLinear(torch.zeros(8, 16), torch.ones(16), torch.zeros(8 * 16 + 16))):
    try:
        call()
    except ImportError as e:
        assert "python -m paper_2506_16235_b200.build" in str(e), e
    else:
        raise AssertionError("the call went through")
print("as expected")
"""


def test_the_package_without_the_module():
    done = subprocess.run([sys.executable, "-c", WITHOUT], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.strip() == "as expected", done.stderr[-2000:]


def test_a_missing_module_alone_is_built_without_the_library(monkeypatch, tmp_path):
    made = []
    monkeypatch.setattr(nsml_build, "NATIVE_PATH", str(tmp_path / "_native.so"))
    monkeypatch.setattr(nsml_build, "_library_is_stale", lambda: False)
    monkeypatch.setattr(nsml_build, "_run", lambda cmd, what, verbose: made.append(what) or open(cmd[cmd.index("-o") + 1], "w").close())
    assert nsml_build.is_stale()
    nsml_build.build()
    assert made == ["_native.so"] and not nsml_build.is_stale()
