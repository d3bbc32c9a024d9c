"""The tree kernels' untracked page-id loads (no GPU; hipcc only): the walk of
test_page_id_register.py over the assembly of tree_attn.hip."""
import os
import re
import subprocess

from paper_2609_36760_amd import build as b
from test_page_id_register import HIPCC, _walk, pytestmark  # noqa: F401


def test_page_id_register_untouched_until_its_wait(tmp_path):
    out = tmp_path / "tree_attn.s"
    r = subprocess.run([HIPCC, *b.HIP_FLAGS, "--cuda-device-only", "-S", os.path.join(b.CSRC, "tree_attn.hip"), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    asm = out.read_text()
    kernels = re.findall(r"^(_ZN\w*decode_kernel\w*):", asm, flags=re.M)
    assert len(kernels) == 10, kernels
    for name in kernels:
        body = asm[asm.index(name + ":"):]
        lines = body[:body.index(".Lfunc_end")].split("\n")
        labels = {l.split(":")[0]: i for i, l in enumerate(lines) if re.match(r"^\.LBB\w+:", l)}
        checked = 0
        for i, l in enumerate(lines):
            m = re.match(r"\s*s_load_dword s(\d+), s\[\d+:\d+\], s\d+\s*$", l.split(";")[0])
            if m:
                bad = _walk(lines, labels, i, int(m.group(1)))
                assert not bad, f"{name}: page id in s{m.group(1)} (line {i}) named before its wait: {bad[:3]}"
                checked += 1
        assert checked >= 4, (name, checked)
