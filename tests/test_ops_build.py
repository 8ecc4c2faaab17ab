"""Build invariants of the operators' kernels, from the compiler's own report: rows of up to 16384 values are held
in registers (no scratch memory), occupancy as the launch counts on, and no packed fp32 arithmetic."""
import os
import re
import subprocess
import tempfile

import pytest

from paper_2603_16428_amd import build as B


@pytest.fixture(scope="module")
def report():
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "ops.s")
        cmd = [B.HIPCC] + [f for f in B.FLAGS if f != "-shared"] + ["-S", "--cuda-device-only",
               "-Rpass-analysis=kernel-resource-usage"] + B.OPS_SOURCES + ["-o", out]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        kernels = {}
        for part in re.split(r"Function Name: ", r.stderr)[1:]:
            kernels[part.split()[0]] = {k: int(re.search(re.escape(k) + r"[^:]*: (\d+)", part).group(1))
                                        for k in ("VGPRs", "ScratchSize", "Occupancy")}
        return kernels, open(out).read()


def _norm(name):
    """(backward, type, threads, steps) of a row kernel's mangled name."""
    m = re.match(r"_ZN3lce\d+(add_rmsnorm(?:_backward)?)_kernelI(DF16b|DF16_|f)Li(\d+)ELi(\d+)E", name)
    return m and ("backward" in m.group(1), m.group(2), int(m.group(3)), int(m.group(4)))


def test_rows_are_in_registers(report):
    kernels, _ = report
    seen = 0
    for name, use in kernels.items():
        n = _norm(name)
        if n is None:
            continue
        seen += 1
        backward, dtype, threads, steps = n
        assert use["ScratchSize"] == 0 or threads == 1024, (name, use)
    # Eleven widths, each with rows that end in whole and in part pieces, and the one for H < 8; three types; the
    # forward in its own type and in e4m3, and the backward.
    assert seen == (2 * 11 + 1) * 3 * 3


def test_gradient_kernels_are_resident_at_once(report):
    """2048 workgroups of 4 waves on 256 CUs of 4 SIMDs: 8 waves each (7 where clipping reads its table from memory)."""
    kernels, _ = report
    names = [n for n in kernels if re.search(r"\d(grad_norm_kernel|grad_norm_many_kernel|clip_kernel|clip_many_kernel)I", n)]
    assert len(names) == 8
    for n in names:
        assert kernels[n]["Occupancy"] >= (7 if "clip_many" in n else 8) and kernels[n]["ScratchSize"] == 0, (n, kernels[n])


def test_no_packed_fp32(report):
    assert not re.search(r"v_pk_(add|mul|fma)_f32", report[1])
