"""What an attention row sees, where its keys lie and how tiles are cut (CPU).

``tests/c_abi/attn_rows_check.hip`` calls the kernels' own functions
(``bsr_attn_rows.h``) on the host and compares them with the definitions on
random requests, and on starts, lengths and block ids out of their ranges:
every row and block table index that a kernel would use stays inside.
"""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_rows_keys_and_parts_match_their_definitions(tmp_path):
    exe = str(tmp_path / "rows")
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", f"-I{ROOT}/include",
                    f"-I{ROOT}/paper_2608_17826_amd/csrc", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", os.path.join(ROOT, "tests", "c_abi", "attn_rows_check.hip"), "-o", exe],
                   check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
