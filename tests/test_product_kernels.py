"""What the built library says of the kernels of the feed-forward products.  Their matrix instructions are written in place, so that the
compiler does not know which instructions they are and keeps none of the distances that the hardware asks for: no sum may be moved to
scratch memory in between, none may be read within eighteen wait states of an instruction that writes it, and no operand may come from a
vector instruction less than two wait states earlier."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2403_04206_amd import buildlib

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
READELF, OBJDUMP = (shutil.which(t) or os.path.join(LLVM, t) for t in ("llvm-readelf", "llvm-objdump"))
pytestmark = pytest.mark.skipif(not os.path.exists(READELF) or not os.path.exists(OBJDUMP), reason="no llvm tools")


@pytest.fixture(scope="module")
def images(tmp_path_factory):
    """The code objects of this library's own kernels: ELF files of machine 224 (AMDGPU) inside its bytes, each up to the next one."""
    if not os.path.exists(buildlib.LIB):
        buildlib.build(force=True)
    data = open(buildlib.LIB, "rb").read()
    starts = [m.start() for m in re.finditer(b"\x7fELF\x02\x01\x01\x40", data)]
    starts = [s for s in starts if int.from_bytes(data[s + 18:s + 20], "little") == 224]
    found = []
    for i, (s, e) in enumerate(zip(starts, starts[1:] + [len(data)])):
        if b"k_gemm" in data[s:e]:
            path = tmp_path_factory.mktemp("image") / ("%d.elf" % i)
            path.write_bytes(data[s:e])
            found.append(str(path))
    assert found
    return found


def test_no_product_kernel_uses_scratch(images):
    seen = {}
    for path in images:
        text = subprocess.run([READELF, "--notes", path], capture_output=True, text=True).stdout
        for name, size in re.findall(r"\.name:\s+(\S+)\n(?:.*\n)*?\s+\.private_segment_fixed_size:\s+(\d+)", text):
            seen[name] = int(size)
    assert len([n for n in seen if "k_gemm" in n]) > 40, sorted(seen)
    assert not {n: s for n, s in seen.items() if s and "k_gemm" in n}


def registers(op):
    m = re.match(r"v\[(\d+):(\d+)\]", op)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    m = re.match(r"v(\d+)$", op)
    return {int(m[1])} if m else set()


def test_distances_around_matrix_instructions(images):
    count = 0
    for path in images:
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], capture_output=True, text=True).stdout
        for body in re.split(r"\n(?=[0-9a-f]+ <)", text):
            name = body.split("\n", 1)[0]
            if "k_gemm" not in name:
                continue
            before = []                                          # (wait states it takes, name, written, read) of what came last
            for line in body.split("\n")[1:]:
                parts = line.split("//")[0].split(None, 1)
                if not parts:
                    continue
                op, ops = parts[0], [o.strip().split()[0] for o in parts[1].split(",") if o.strip()] if len(parts) > 1 else []
                valu, mfma = op.startswith("v_"), op.startswith("v_mfma")
                writes = registers(ops[0]) if valu and ops and not op.startswith("v_cmp") else set()
                reads = set().union(*[registers(o) for o in (ops[1:] if valu else ops)]) if ops else set()
                states = 0
                for took, op2, writes2 in reversed(before):
                    if op2.startswith("v_mfma"):
                        assert mfma or states >= 18 or not writes2 & (reads | writes), (name, line, "after", op2)
                    elif mfma:
                        assert states >= 2 or not writes2 & reads, (name, line, "after", op2)
                    states += took
                    if states > 18:
                        break
                count += mfma
                before.append((int(ops[0]) + 1 if op == "s_nop" else 1, op, writes))
                del before[:-24]
    assert count > 4000
