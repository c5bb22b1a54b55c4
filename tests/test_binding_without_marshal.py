"""The binding where the extension module cannot be loaded: the entries that do not need it work, the others say what is missing."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import sys
sys.modules["paper_2608_13057_b200._marshal"] = None             # as if the module were not there
import torch
from paper_2608_13057_b200 import binding as B
from paper_2608_13057_b200 import layer
s = B.make_shape(4, 2, 8, 2, 1, 128, 128, 128)
assert B.tempo_version() >= 1 and B.tempo_m_cap_bound(s) == 384 and B.tempo_few_workspace_bytes(s) > 0
try:
    B.tempo_permute_pad(s, *[torch.zeros(1)] * 6)
    raise SystemExit("accepted")
except B.TempoError as e:
    assert "CUDA tensor" in str(e)
r = torch.zeros(4, 128)
for call in (lambda: B.tempo_norm_in(r, r[0], r), lambda: B.tempo_norm_out(r, r, r), lambda: B.tempo_route(s, r, r, None, None, r, r, r),
             lambda: B.tempo_few_ffn(s, r, r, r, None, r, r, r, r, r), lambda: B.tempo_few_ffn_bf16(s, r, r, r, None, r, r, r, r, r)):
    try:
        call()
        raise SystemExit("accepted")
    except ImportError as e:
        assert "_marshal" in str(e) and "build" in str(e), e
print("fine")
"""


def test_entries_without_the_extension_module():
    from paper_2608_13057_b200 import build
    build.build()
    res = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True)
    assert res.returncode == 0 and "fine" in res.stdout, res.stderr[-2000:]
