"""Where the attention kernels over the 8-bit cache use scratch (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2604_03957_amd import build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _bodies(path):
    """{mangled kernel name: its assembly lines}"""
    out, name = {}, None
    for line in open(path):
        m = re.match(r"(_Z\S*k_cache_attention\S*):", line)
        if m:
            name = m.group(1)
            out[name] = []
        elif line.startswith(".Lfunc_end"):
            name = None
        elif name:
            out[name].append(line.rstrip())
    return out


def _step_loop(lines):
    """The lines of the smallest loop around at least eight matrix instructions: a step over 64 keys."""
    labels = {line.split(":")[0]: n for n, line in enumerate(lines) if line.startswith(".LBB")}
    loops = []
    for n, line in enumerate(lines):
        m = re.search(r"s_c?branch\S*\s+(\.LBB\S+)", line)
        if m and labels.get(m.group(1), n) < n:
            body = lines[labels[m.group(1)]:n]
            if sum("v_mfma" in x for x in body) >= 8:
                loops.append(body)
    return min(loops, key=len)


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_scratch_of_the_attention_kernels_stays_outside_their_steps(tmp_path):
    """Many rows of heads of 128 need some registers more than there are: what lies in scratch is read at a tile's beginning and end.
    Inside a step an access to it would wait for the codes that are on their way."""
    s = tmp_path / "attention.s"
    cmd = [HIPCC] + build.HIPCC_FLAGS + ["--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-S", os.path.join(build.CSRC, "kernels_cache_attention.hip"), "-o", str(s)]
    report = subprocess.run(cmd, stderr=subprocess.PIPE, text=True, check=True).stderr
    names = re.findall(r"Function Name: (\S+)", report)
    scratch = dict(zip(names, (int(b) for b in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", report))))
    bodies = {n: b for n, b in _bodies(s).items() if "join" not in n}
    assert len(bodies) == 32 and set(bodies) <= set(scratch)
    for name, lines in bodies.items():
        step = _step_loop(lines)
        assert sum("v_mfma" in x for x in step) >= 16, name
        assert not [x for x in step if "scratch_" in x], name
    # bytes a lane: what the comments beside the kernels say
    some = {re.sub(r"^_ZN4bwta12_GLOBAL__N_1\d\d|EEEvNS_.*$", "", n): b for n, b in scratch.items() if b}
    assert set(some) == {"k_cache_attention%s" % x for t in ("DF16_", "DF16b") for x in
                         ("_rowsI%sLi128ELi1ELb0" % t, "_rowsI%sLi128ELi1ELb1" % t, "_rowsI%sLi128ELi2ELb0" % t, "I%sLi128ELi2ELi8" % t)}
    assert max(some.values()) <= 56
