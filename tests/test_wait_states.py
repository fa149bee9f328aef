"""What the hardware asks of instruction sequences that inline assembly puts together, looked up in the built library's own code (no GPU needed): a scalar register
that a vector instruction has written is good for a memory instruction five wait states later (one per instruction, s_nop n: n + 1).  The compiler keeps to
that for its own instructions and does not look into inline assembly."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2603_21365_amd.build import LIB_PATH

LLVM = "/opt/rocm/llvm/bin"


def kernels(tmp_path):
    """(kernel, its instructions) of the library's gfx950 code."""
    tools = {t: os.path.join(LLVM, t) if os.path.exists(os.path.join(LLVM, t)) else shutil.which(t) for t in ("llvm-objcopy", "clang-offload-bundler", "llvm-objdump")}
    if not all(tools.values()):
        pytest.skip("the toolchain's binary tools are not here")
    if not os.path.exists(LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.run([tools["llvm-objcopy"], f"--dump-section=.hip_fatbin={fat}", LIB_PATH, str(tmp_path / "rest")], check=True)
    targets = subprocess.run([tools["clang-offload-bundler"], "--list", "--type=o", f"--input={fat}"], check=True, capture_output=True, text=True).stdout.split()
    target = next(t for t in targets if "gfx950" in t)
    subprocess.run([tools["clang-offload-bundler"], "--unbundle", "--type=o", f"--input={fat}", f"--targets={target}", f"--output={code}"], check=True)
    text = subprocess.run([tools["llvm-objdump"], "-d", "--no-show-raw-insn", "--no-leading-addr", code], check=True, capture_output=True, text=True).stdout
    name, body = None, []
    for line in text.splitlines():
        start = re.match(r"^(?:[0-9a-f]+ )?<(\S+)>:$", line)
        if start:
            if name:
                yield name, body
            name, body = start.group(1), []
        elif line.startswith("\t") and name:
            body.append(line.split("//")[0].strip())
    yield name, body


def scalars(text):
    out = set()
    for a, b, c in re.findall(r"\bs\[(\d+):(\d+)\]|\bs(\d+)\b", text):
        out |= set(range(int(a or c), int(b or c) + 1))
    return out


def too_soon(body):
    """(waited, writer, reader) where a memory instruction reads a scalar register less than five wait states after a vector instruction wrote it."""
    found = []
    for at, text in enumerate(body):
        if not re.match(r"(buffer|global|flat|scratch)_", text):
            continue
        need, waited = scalars(text), 0
        for before in reversed(body[max(0, at - 5):at]):
            if waited >= 5 or not need:
                break
            writer = re.match(r"v_(?:readfirstlane|readlane|cmp)\S*\s+(s\[\d+:\d+\]|s\d+)", before)
            if writer and need & scalars(writer.group(1)):
                found.append((waited, before, text))
            nops = re.match(r"s_nop (\d+)", before)
            waited += 1 + (int(nops.group(1)) if nops else 0)
    return found


def test_the_search_finds_what_it_looks_for():
    load = "buffer_load_dwordx4 v2, s[8:11], 0 offen lds"
    assert too_soon(["v_readfirstlane_b32 s10, v1", "s_mov_b32 m0, s4", "s_nop 0", load])
    assert too_soon(["v_cmp_gt_u32_e64 s[10:11], v1, v2", "s_nop 3", load])
    assert not too_soon(["v_readfirstlane_b32 s10, v1", "s_nop 4", "s_mov_b32 m0, s4", "s_nop 0", load])
    assert not too_soon(["v_readfirstlane_b32 s12, v1", load])


def test_memory_instructions_wait_for_their_scalar_registers(tmp_path):
    seen, loads, bad = 0, 0, {}
    for name, body in kernels(tmp_path):
        seen += 1
        loads += sum(bool(re.match(r"buffer_load_dwordx4 .* lds", t)) for t in body)
        found = too_soon(body)
        if found:
            bad[name] = found
    assert seen > 50 and loads > 500, (seen, loads)
    assert not bad, f"{sum(map(len, bad.values()))} in {len(bad)} kernels: {next(iter(bad.items()))}"
