"""The causal backward issues score and update products from assembly statements, as the bidirectional one does: the same check of
its emitted assembly (tests/isa_lint.py) that no result is read too early."""
import os
import subprocess

from paper_2503_12964_amd import build
from tests import isa_lint as L


def test_causal_backward_kernels_keep_the_rule(tmp_path):
    out = tmp_path / "cattn_bwd.s"
    cmd = [build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "cattn_bwd.hip"), "-o", str(out)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    text = out.read_text()
    prog = L.parse(text)
    assert sum(1 for i in prog.insts if i.from_asm and i.mnemonic.startswith("v_mfma")) >= 300     # (the markers were recognised)
    bad = L.check(text)
    assert bad == [], "\n".join(bad[:20])
