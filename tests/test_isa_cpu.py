"""Required distances between instructions in the built library.  The compiler keeps them for what it selects itself; the result of
inline assembly it does not count as a vector operation's, so nothing but the schedule separates it from an instruction that needs
wait states behind such a result.  No GPU is needed: the library's own gfx950 code is disassembled."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2510_05176_amd", "libpatternkv.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"

pytestmark = pytest.mark.skipif(not os.path.exists(LIB) or not os.path.exists(OBJDUMP), reason="no built library or no disassembler")


def _registers(text):
    out = set()
    for one, lo, hi in re.findall(r"\bv(\d+)\b|\bv\[(\d+):(\d+)\]", text):
        out |= {int(one)} if one else set(range(int(lo), int(hi) + 1))
    return out


def _too_close(asm, needed=2):
    """(reads of the three kinds, those with fewer than `needed` wait states behind the vector operation that wrote them)"""
    kernel, seen, bad, recent = None, {"lane swap": 0, "lane permutation": 0, "matrix": 0}, [], []
    for line in asm.splitlines():
        line = line.split("//")[0].strip()
        start = re.match(r"^[0-9a-f]* ?<(.*)>:", line)
        if start:
            kernel, recent = start.group(1), []
            continue
        op, _, rest = line.partition(" ")
        if not op or not re.match(r"[a-z]+_", op):
            continue
        operands = [o.strip() for o in rest.split(",")]
        swap, matrix = op.startswith("v_permlane"), op.startswith("v_mfma")
        kind, reads = None, set()
        if swap:
            kind, reads = "lane swap", _registers(rest)
        elif matrix:
            kind, reads = "matrix", _registers(",".join(operands[1:]))
        elif re.search(r"\b(quad_perm|row_\w+|wave_\w+):|\brow_(half_)?mirror\b", rest):
            kind, reads = "lane permutation", _registers(operands[1].split(" ")[0])
        if kind:
            seen[kind] += 1
            for written, distance, by in recent:
                if written & reads and distance < needed:
                    bad.append((kernel, kind, distance, by, line))
                    break
        step = 1 + int(rest) if op == "s_nop" else 1
        recent = [(w, d + step, by) for w, d, by in recent if d + step < needed]
        if op.startswith("v_") and not matrix and not op.startswith(("v_cmp", "v_readlane", "v_readfirstlane", "v_dot")):
            recent.insert(0, (_registers(operands[0]) | (_registers(operands[1]) if "swap" in op else set()), 0, line))
    return seen, bad


def test_the_check_sees_a_missing_wait():
    head = "0 <kernel>:\n v_max_f32_e32 v5, v5, v6\n"
    assert len(_too_close(head + " v_permlane32_swap_b32_e32 v4, v5\n")[1]) == 1
    assert len(_too_close(head + " s_nop 0\n v_permlane32_swap_b32_e32 v4, v5\n")[1]) == 1
    assert len(_too_close(head + " s_nop 1\n v_permlane32_swap_b32_e32 v4, v5\n")[1]) == 0
    assert len(_too_close(head + " v_mov_b32_e32 v1, v2\n v_mfma_f32_16x16x32_f16 v[0:3], v[4:7], v[8:11], v[0:3]\n")[1]) == 1
    assert len(_too_close(head + " v_mov_b32_dpp v1, v5 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n")[1]) == 1


def test_vector_results_are_not_read_too_early(tmp_path):
    """Two wait states from a vector operation to a lane swap, a permuted operand or a matrix operation that reads its result."""
    shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    images = [f for f in sorted(os.listdir(tmp_path)) if f.endswith("gfx950") and os.path.getsize(tmp_path / f)]
    assert images
    total, bad = {}, []
    for f in images:
        r = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", "--no-leading-addr", f], cwd=tmp_path, check=True,
                           capture_output=True, text=True)
        seen, found = _too_close(r.stdout)
        bad += found
        total = {k: total.get(k, 0) + n for k, n in seen.items()}
    assert all(total.values()), total
    assert not bad, (len(bad), bad[:4])


def _arrives_without_a_barrier(asm):
    """Of every kernel in the listing (branch targets as labels): whether an atomic on memory can be reached from its start past no barrier."""
    out = {}
    for name, body in re.findall(r"^[0-9a-f]* ?<([^>]*)>:\n(.*?)(?=^[0-9a-f]* ?<_Z|\Z)", asm, re.M | re.S):
        lines = [x.split("//")[0].strip() for x in body.splitlines()]
        label = {m.group(1): i for i, x in enumerate(lines) if (m := re.match(r"^[0-9a-f]* ?<(L\d+)>:", x))}
        todo, seen, out[name] = [0], set(), False
        while todo:
            i = todo.pop()
            if i in seen or i >= len(lines):
                continue
            seen.add(i)
            op, _, to = lines[i].partition(" ")
            assert not op.startswith(("s_setpc", "s_swappc", "s_call")), lines[i]
            out[name] |= op.startswith(("global_atomic", "flat_atomic", "buffer_atomic"))
            if op == "s_barrier" or op == "s_endpgm":
                continue
            if op.startswith(("s_cbranch", "s_branch")):
                todo.append(label[to.strip()])
            if op != "s_branch":
                todo.append(i + 1)
    return out


def test_the_check_sees_a_missing_barrier():
    head = "0 <_Zkernel>:\n s_load_dword s2, s[0:1], 0x0\n s_cbranch_scc0 L0\n s_barrier\n s_branch L1\n0 <L0>:\n v_nop\n%s0 <L1>:\n global_atomic_add v0, v1, v2, s[0:1]\n s_endpgm\n"
    assert _arrives_without_a_barrier(head % "") == {"_Zkernel": True}
    assert _arrives_without_a_barrier(head % " s_barrier\n") == {"_Zkernel": False}


def test_append_counts_a_workgroup_when_all_its_waves_have_the_state(tmp_path):
    """An append in place replaces the state that its launch reads, once every workgroup of the sequence is counted as arrived.  One wave counts
    for its workgroup, so on every way there, with a block of vectors or without one, it passes a barrier behind the loads of the
    others (64 channels in blocks of 32 tokens have workgroups of one wave)."""
    shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    found = {}
    for f in sorted(os.listdir(tmp_path)):
        if f.endswith("gfx950") and b"fp8_append_kernel" in (tmp_path / f).read_bytes():
            r = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", "--symbolize-operands", f], cwd=tmp_path, check=True,
                               capture_output=True, text=True)
            found.update({k: v for k, v in _arrives_without_a_barrier(r.stdout).items() if "fp8_append_kernel" in k})
    assert len(found) == 24
    assert [k for k, v in found.items() if v and "ILi64ELi32E" not in k] == []


def _lds_requests(asm):
    """(loads from memory to LDS, those that are not a wait state or more behind a scalar instruction that wrote m0 in the same run of instructions)"""
    seen, bad, kernel, since, by = 0, [], None, None, None
    for line in asm.splitlines():
        line = line.split("//")[0].strip()
        start = re.match(r"^[0-9a-f]* ?<(.*)>:", line)
        if start:
            kernel = kernel if re.fullmatch(r"L\d+", start.group(1)) else start.group(1)
            since = by = None   # (a branch may come from anywhere)
            continue
        op, _, rest = line.partition(" ")
        if not op or not re.match(r"[a-z]+_", op):
            continue
        if re.match(r"(global|buffer)_load_lds|buffer_load.*\blds\b", line):
            seen += 1
            if since is None or since < 1 or not by.startswith("s_"):
                bad.append((kernel, by, since, line))
        if re.match(r"m0\b", rest):
            since, by = 0, op
        elif since is not None:
            since += 1 + int(rest) if op == "s_nop" else 1
    return seen, bad


def test_the_check_sees_a_missing_m0():
    load = " global_load_lds_dwordx4 v1, s[0:1]\n"
    assert _lds_requests("0 <_Zkernel>:\n s_mov_b32 m0, s4\n s_nop 0\n" + load) == (1, [])
    assert _lds_requests("0 <_Zkernel>:\n s_add_i32 m0, s4, 0x400\n v_mov_b32_e32 v1, v2\n" + load) == (1, [])
    for before in ("", " s_mov_b32 m0, s4\n", " v_readfirstlane_b32 m0, v4\n s_nop 0\n", " s_mov_b32 m0, s4\n s_nop 0\n0 <L0>:\n"):
        assert len(_lds_requests("0 <_Zkernel>:\n" + before + load)[1]) == 1


def test_loads_to_lds_have_their_place(tmp_path):
    """A load from memory to LDS takes its place from m0, which a scalar instruction writes one wait state or more before it."""
    shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    total, bad = 0, []
    for f in sorted(os.listdir(tmp_path)):
        if f.endswith("gfx950") and b"prompt_kernel" in (tmp_path / f).read_bytes():
            r = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", "--symbolize-operands", f], cwd=tmp_path, check=True,
                               capture_output=True, text=True)
            seen, found = _lds_requests(r.stdout)
            total, bad = total + seen, bad + found
    assert total > 0
    assert not bad, (len(bad), bad[:4])


def test_no_assembly_writes_m0_behind_the_compilers_back():
    """m0 is a reserved register, which no list of clobbers takes; as an operand ("{m0}") the compiler writes it itself and knows of it."""
    csrc, found = os.path.join(ROOT, "paper_2510_05176_amd", "csrc"), []
    for f in sorted(os.listdir(csrc)):
        with open(os.path.join(csrc, f)) as text:
            for statement in re.findall(r"\basm\b(?:\s+volatile)?\s*\((.*?)\);", text.read(), re.S):
                template = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', statement.split(" : ", 1)[0]))
                if re.search(r"\bm0\b", template.replace("\\n", "\n").replace("\\t", "\t")):
                    found.append((f, template))
    assert not found, found
