"""The clamp of a verify call's lengths keeps every 32-bit key number and the sum of all tiles in range, and leaves what
fits alone."""
import os
import shutil
import subprocess

import pytest

from paper_2504_06419_amd import build

PROGRAM = r"""
#include <stdio.h>
#include "spire_internal.h"
int main() {
    for (int paged = 0; paged < 2; ++paged)
        for (long cap = 1; cap < (1l << 45); cap = cap * 3 + 1)
            for (int B : {0, 1, 2, 3, 64, 1000, 8191, 8192}) {
                spire::KvDev kv = {};
                if (paged) { kv.page_size = 16; kv.max_blocks = (int)((cap + 15) / 16 < INT32_MAX ? (cap + 15) / 16 : INT32_MAX); }
                else kv.capacity = (int)(cap < INT32_MAX ? cap : INT32_MAX);
                printf("%ld %d %d\n", paged ? 16l * kv.max_blocks : (long)kv.capacity, B, spire::most_keys(kv, B));
            }
}
"""


@pytest.mark.skipif(not os.path.exists(build._hipcc()), reason="needs hipcc")
def test_clamp(tmp_path):
    (tmp_path / "a.hip").write_text(PROGRAM)
    subprocess.run([build._hipcc(), *build.FLAGS, "-I", build.CSRC, "-I", os.path.join(build.CSRC, "..", "..", "include"),
                    str(tmp_path / "a.hip"), "-o", str(tmp_path / "a")], check=True, capture_output=True)
    out = subprocess.run([str(tmp_path / "a")], check=True, capture_output=True, text=True).stdout
    rows = [tuple(map(int, ln.split())) for ln in out.splitlines()]
    assert len(rows) > 300
    for cap, B, most in rows:
        assert 1 <= most <= cap and most + 63 * 64 + 64 < 2**31          # the copies look 63 tiles of 64 keys ahead
        assert B * (-(-most // 16) + 1000) < 2**31                       # the positions' prefix sums
        if cap <= 2**22 - 2**14 - 64 or (B <= 1 and cap <= 2**31 - 8192):
            assert most == cap
