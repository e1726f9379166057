"""The machine code of the kernels, as built: where lanes that took a branch and those that did not come together again, no vector instruction stands before the one that lets all lanes run.

Under register pressure the compiler has placed copies of live registers there: they ran for the lanes of the branch alone, and the others read the old registers from then on, as addresses
among others.  The sources avoid such branches where registers are scarce; this looks at what became of them."""
import os
import re
import subprocess

import pytest

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
VECTOR = ("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")
SCALAR_RESULT = ("v_readlane", "v_writelane", "v_readfirstlane")      # (of a lane that is named, or of any: no lane's own register)


def early(text):
    """[(kernel, label, instructions)]: vector instructions between the head of a block that branches with an empty mask go to, and its `s_or_b64 exec`"""
    targets = set(re.findall(r"s_cbranch_execz (L\d+)", text))
    found, kernel, label, before, open_ = [], None, None, [], False
    for line in text.splitlines():
        head = re.match(r"<(.+)>:", line)
        if head:
            name = head.group(1)
            if re.fullmatch(r"L\d+", name):
                label, open_ = name, name in targets
            else:
                kernel, label, open_ = name, None, False
            before = []
            continue
        code = line.split("//")[0].strip()
        if not code:
            continue
        op = code.split()[0]
        if op == "s_cbranch_execnz":      # (what follows a loop whose lanes leave one by one)
            label, before, open_ = "behind a loop", [], True
        elif open_:
            if re.match(r"s_or_b64 exec, exec", code):
                if before:
                    found.append((kernel, label, before))
                open_ = False
            elif op.startswith(("s_cbranch", "s_branch", "s_endpgm")) or "saveexec" in op:
                open_ = False
            elif op.startswith(VECTOR) and not op.startswith(SCALAR_RESULT):
                before.append(code)
    return found


def test_what_is_looked_for():
    body = "<kernel>:\n\ts_and_saveexec_b64 s[0:1], vcc  // 0: 1\n\ts_cbranch_execz L0  // 4: 2\n\tglobal_store_dword v[0:1], v2, off\n<L0>:\n%s\ts_or_b64 exec, exec, s[0:1]\n\tv_add_u32 v0, v1, v2\n\ts_endpgm\n"
    assert early(body % "") == [] and early(body % "\ts_mov_b32 s2, 0\n\tv_readlane_b32 s3, v9, 1\n") == []
    assert early(body % "\tv_mov_b32_e32 v242, v93  // 8: 3\n") == [("kernel", "L0", ["v_mov_b32_e32 v242, v93"])]


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler of this library's own code here")
def test_no_vector_instruction_before_the_lanes_are_back(tmp_path):
    import paper_2501_09849_amd.build as build
    if not os.path.exists(build.LIB_PATH):
        build.build_lib()
    os.symlink(build.LIB_PATH, tmp_path / "libcdl.so")
    subprocess.run([OBJDUMP, "--offloading", "libcdl.so"], cwd=tmp_path, check=True, capture_output=True)
    kernels = branches = 0
    for name in sorted(os.listdir(tmp_path)):
        if "amdgcn" not in name:
            continue
        text = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn", "--no-leading-addr", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        kernels += len(re.findall(r"^<_Z.+>:", text, re.M))
        branches += len(re.findall(r"s_cbranch_execz L\d+", text))
        assert early(text) == [], name
    assert kernels > 100 and branches > kernels      # (the listing is as it is read here)
