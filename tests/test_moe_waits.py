"""The waits of the experts' products' kernels, read from the built code as those
of the products of one weight are: at a barrier after which other waves write a
stage of LDS, no read of that stage may still be under way."""
import re
import subprocess

import pytest

import paper_2003_04296_amd as q
from test_dense_waits import OBJDUMP, _under_way
from test_kernel_registers import _code_objects


def _kernels(tmp_path):
    for i, obj in enumerate(_code_objects(q.LIB_PATH)):
        if b"moe_gemm_kernel" not in obj:
            continue
        f = tmp_path / f"{i}.co"
        f.write_bytes(obj)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(f)], check=True,
                              capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]* ?<\S+>:\n)", text):
            head, _, body = part.partition("\n")
            name = re.search(r"<(\S+)>:", head)
            if name and re.search("moe_gemm(_w)?_kernel", name.group(1)):
                yield name.group(1), body.split("\n")


@pytest.mark.skipif(OBJDUMP is None, reason="llvm-objdump reads the kernels")
def test_reads_have_ended_at_barriers(tmp_path):
    found = dict(_kernels(tmp_path))
    assert len(found) == 24
    for name, lines in found.items():
        # products a stage, whether in column form, whether straight into LDS
        m = re.search(r"Stage16ILi(\d+)ELi\d+ELi\d+ELi0ELb([01])ELb([01])E", name)
        at = _under_way(lines)
        assert at, name
        early = 0
        if m.group(1) == "32" and m.group(3) == "1":
            # 3 row fragments and 4 column fragments of the next stage, which is
            # written again one barrier later; two reads each in column form
            early = 3 * (2 if m.group(2) == "1" else 1) + 4 * 2
        assert max(at) <= early, (name, at)
