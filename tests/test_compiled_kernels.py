"""Two faults of the compiler (ROCm 7.2) that the sources are written around, looked for in the built kernels (no GPU):

- copies of live values in a block where masked lanes come together again, in front of the instruction that gives those lanes back: only
  the lanes of one side are copied, the others come back with whatever the target held, addresses among it;
- a matrix instruction's result read, behind a branch, sooner than the 8 cycles that the compiler keeps within a block."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2202_05239_amd import binding as f8

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
WAIT = 8
COPY = re.compile(r"v_accvgpr_|v_mov_b(32|64)(_e32|_e64)? v\S+ v|scratch_")


def registers(text):
    out = set()
    for m in re.finditer(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out |= {(m.group(1), i) for i in range(int(m.group(2) or m.group(4)), int(m.group(3) or m.group(4)) + 1)}
    return out


def operands(t):
    return t.split(None, 1)[1] if " " in t else ""


class Kernel:
    """A kernel's instructions, and those that may follow each of them."""

    def __init__(self, code):
        self.text, at = [t for _, t in code], {a: i for i, (a, _) in enumerate(code)}
        self.next = []
        for i, (a, t) in enumerate(code):
            to = [i + 1] if i + 1 < len(code) else []
            if t.startswith(("s_branch", "s_cbranch")):
                words = int(t.split()[1])
                target = at[a + 4 + 4 * (words - 65536 if words >= 32768 else words)]
                to = [target] if t.startswith("s_branch") else to + [target]
            self.next.append([] if t.startswith("s_endpgm") else to)

    def misplaced_copies(self):
        """Copies between the start of a block that ends a branch or a loop over lanes and the instruction that gives the lanes back."""
        found, starts, masked = [], set(), None
        for i, t in enumerate(self.text):
            if "saveexec" in t or t.startswith("s_andn2_b64 exec, exec"):
                masked = i
            elif t.startswith(("s_branch", "s_cbranch")):
                if masked is not None and i - masked <= 4 and t.startswith("s_cbranch_exec"):
                    starts.add(self.next[i][1 if t.startswith("s_cbranch_execz") else 0])
                masked = None
        for i in starts:
            copies = []
            for t in self.text[i:]:
                if re.match(r"s_or_b64 exec, exec|s_\w*saveexec", t):
                    found += copies
                    break
                if re.match(r"s_(c?branch|endpgm)|s_\w+ exec\b", t):
                    break
                if COPY.match(t):
                    copies.append(t)
        return found

    def early_reads(self):
        """(cycles at least, matrix instruction, reader) of results that are used within WAIT on some path, by others than products."""
        found = []
        for i, t in enumerate(self.text):
            if not t.startswith("v_mfma"):
                continue
            result, best, stack = registers(operands(t).split(",")[0]), {}, [(j, 0) for j in self.next[i]]
            while stack:
                j, waited = stack.pop()
                if waited >= WAIT or best.get(j, WAIT) <= waited:
                    continue
                best[j], u = waited, self.text[j]
                if u.startswith("v_mfma"):
                    if registers(operands(u).split(",")[0]) & result:         # (a sum that goes on has a wait of its own)
                        continue
                    waited += 4
                elif u.startswith("s_nop"):
                    waited += int(operands(u)) + 1
                elif registers(operands(u)) & result:
                    found.append((waited, t, u))
                    continue
                else:
                    waited += 1
                stack += [(k, waited) for k in self.next[j]]
        return found


def parse(lines):
    kernels, code = {}, None
    for line in lines:
        m = re.match(r"^[0-9a-f]{16} <(\S+)>:", line)
        if m:
            code = kernels.setdefault(m.group(1), [])
        elif code is not None and "// 0" in line:
            text, _, address = line.partition("//")
            code.append((int(address.split(":")[0], 16), text.strip()))
    return {name: Kernel(code) for name, code in kernels.items() if code}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    where = tmp_path_factory.mktemp("code")
    shutil.copy(f8.LIB_PATH, where / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=where, check=True, capture_output=True)
    out = {}
    for name in sorted(os.listdir(where)):
        if name.endswith("gfx950"):
            run = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", name], cwd=where, check=True, capture_output=True, text=True)
            out.update(parse(run.stdout.split("\n")))
    return out


def test_no_copy_in_front_of_the_lanes(kernels):
    assert sum("attend_shared_kernel" in name for name in kernels) == 12
    assert {name: k.misplaced_copies()[:3] for name, k in kernels.items() if k.misplaced_copies()} == {}


def test_results_of_matrix_instructions_are_waited_for(kernels):
    assert sum(any(t.startswith("v_mfma") for t in k.text) for k in kernels.values()) > 100
    assert {name: early[:3] for name, early in ((name, k.early_reads()) for name, k in kernels.items()) if early} == {}


def test_both_are_found_where_they_are():
    def kernel(*text):
        return next(iter(parse(["0000000000000000 <k>:"] + ["\t%s  // %012X: 0" % (t, 4 * i) for i, t in enumerate(text)]).values()))
    masked = ("v_cmp_gt_u32_e32 vcc, 4, v0", "s_and_saveexec_b64 s[2:3], vcc", "s_cbranch_execz 1", "v_add_u32_e32 v1, 1, v1")
    assert kernel(*masked, "s_or_b64 exec, exec, s[2:3]", "v_mov_b32_e32 v7, v6", "s_endpgm").misplaced_copies() == []
    assert kernel(*masked, "v_mov_b32_e32 v7, v6", "s_or_b64 exec, exec, s[2:3]", "s_endpgm").misplaced_copies() == ["v_mov_b32_e32 v7, v6"]
    product = "v_mfma_f32_16x16x32_f16 v[4:7], v[8:11], v[12:15], v[4:7]"
    for nops, early in ((6, 0), (5, 1)):                                     # one instruction, s_nop n is n + 1, the branch is one
        got = kernel(product, "v_add_u32_e32 v1, 1, v1", "s_nop %d" % (nops - 1), "s_cbranch_scc1 1", "s_endpgm", "v_mul_f32_e32 v2, v5, v3", "s_endpgm").early_reads()
        assert len(got) == early
    assert kernel(product, product, "s_endpgm").early_reads() == []
