"""LDS of the attention kernels, in the assembly that this build makes of them: what a launch asks for is what the workgroups write.
Panels and rows' statistics are filled by loads straight into LDS; the only stores are those of the common part of the keys in the bf16
backward pass."""
import re
import subprocess

import pytest

from paper_2607_19331_amd import build as B


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("attend_lds") / "grad.s"
    subprocess.run(["hipcc", *B.HIPFLAGS, "-x", "hip", "-S", "--cuda-device-only", f"{B.CSRC}/iso_attend_grad.hip", "-o", str(out)],
                   check=True, capture_output=True)
    text = out.read_text()
    return {(int(m[1]), int(m[2])): m[3]
            for m in re.finditer(r"^\S*k_attend_gradILi(\d)ELi(\d+)E\S*:.*?\n(.*?)\.Lfunc_end", text, re.S | re.M)}


def stores(text):
    return [line.strip() for line in text.splitlines() if re.match(r"\s*ds_(write|store|add|min|max|wrxchg)", line)]


@pytest.mark.parametrize("dim", [64, 128])
def test_fp32_workgroups_store_nothing_behind_their_panels(kernels, dim):
    """Their launch asks for the panels and 512 bytes that loads fill."""
    assert "buffer_load_dwordx4" in kernels[0, dim]
    assert stores(kernels[0, dim]) == []
