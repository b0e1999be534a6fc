"""Host-side check of the built kernels for the same two hazards as test_memory_hazards.py, along every way that execution can take: over the back edges of loops and into either side
of a branch; with whatever vector instruction writes a scalar register, and stores whose data are accumulators.  The objects were compiled here; no GPU needed."""
import glob
import os
import re
import shutil
import subprocess

import pytest

LLVM = "/opt/rocm/llvm/bin"


class Code:
    """A kernel's instructions as (name, operands), and of each the places that it may be followed by."""

    def __init__(self, lines):
        self.ops, self.next, at, jumps = [], [], {}, {}
        for line in lines:
            text, _, note = line.partition("//")
            if not text.strip():
                continue
            name, _, rest = text.strip().partition(" ")
            where = re.match(r"\s*([0-9A-F]{6,}):", note)
            if where:
                at[int(where.group(1), 16)] = len(self.ops)
            if name.startswith(("s_cbranch", "s_branch")):
                to = int(rest.split()[0])
                jumps[len(self.ops)] = int(where.group(1), 16) + 4 + 4 * (to - 65536 if to > 32767 else to)
            self.ops.append((name, rest.strip()))
        for i, (name, _) in enumerate(self.ops):
            ends = name.startswith(("s_endpgm", "s_branch", "s_setpc", "s_swappc"))
            to = [] if ends or i + 1 == len(self.ops) else [i + 1]
            self.next.append(to + ([at[jumps[i]]] if i in jumps else []))

    def reached(self, i, states):
        """The instructions that execution can come to with fewer than `states` wait states between them and instruction i."""
        seen, todo = {}, [(j, 0) for j in self.next[i]]
        while todo:
            j, ago = todo.pop()
            if ago >= states or seen.get(j, states) <= ago:
                continue
            seen[j] = ago
            name, rest = self.ops[j]
            ago += int(rest, 0) + 1 if name == "s_nop" else 1
            todo += [(k, ago) for k in self.next[j]]
        return seen


def _registers(text, kind):
    out = set()
    for lo, hi in re.findall(r"\b" + kind + r"\[(\d+):(\d+)\]", text):
        out |= set(range(int(lo), int(hi) + 1))
    out |= {int(n) for n in re.findall(r"\b" + kind + r"(\d+)\b", text)}
    if kind == "s":
        out |= {106, 107} if re.search(r"\bvcc\b", text) else {106} if "vcc_lo" in text else {107} if "vcc_hi" in text else set()
    return out


MEMORY = ("buffer_", "global_", "flat_", "scratch_")


def scalars_written(name, rest):
    """Scalar registers that a vector instruction writes."""
    parts = rest.split(", ")
    if name.startswith("v_cmp"):
        return _registers(parts[0], "s") or {106, 107}
    if name.startswith(("v_readlane", "v_readfirstlane")):
        return _registers(parts[0], "s")
    if "_co_" in name or name.startswith(("v_div_scale", "v_mad_u64_u32", "v_mad_i64_i32")):
        return _registers(parts[1], "s")
    return set()


def scalars_not_there_yet(code):
    """Memory instructions that can read a scalar register fewer than five wait states after a vector instruction wrote it."""
    bad = []
    for i, (name, rest) in enumerate(code.ops):
        written = scalars_written(name, rest) if name.startswith("v_") else None
        if written:
            bad += [(i, j) for j in code.reached(i, 5) if code.ops[j][0].startswith(MEMORY) and written & _registers(code.ops[j][1], "s")]
    return bad


def data_overwritten(code):
    """Stores of more than eight bytes whose data a vector instruction can write within the next two wait states."""
    bad = []
    for i, (name, rest) in enumerate(code.ops):
        if not re.match(r"(buffer|global|flat|scratch)_store_dwordx[34]", name):
            continue
        data = rest.split(", ")[0 if name.startswith("buffer") else 1]
        for j in code.reached(i, 2):
            after, operands = code.ops[j]
            if after.startswith("v_") and not after.startswith(("v_readlane", "v_readfirstlane", "v_cmp")):
                to = operands.split(", ")[0]
                if any(_registers(data, kind) & _registers(to, kind) for kind in "va"):
                    bad.append((i, j))
    return bad


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    import paper_2505_24791_amd as sjd
    if not os.path.exists(sjd.LIB_PATH):
        from paper_2505_24791_amd import build
        build.build()
    d = tmp_path_factory.mktemp("objects")
    shutil.copy(sjd.LIB_PATH, d / "libsjd.so")
    subprocess.run([f"{LLVM}/llvm-objdump", "--offloading", "libsjd.so"], cwd=d, check=True, stdout=subprocess.DEVNULL)
    found = {}
    for obj in glob.glob(str(d / "*gfx950")):
        text = subprocess.run([f"{LLVM}/llvm-objdump", "-d", "--no-show-raw-insn", obj], check=True, stdout=subprocess.PIPE, text=True).stdout
        for part in re.split(r"^[0-9a-f]+ <", text, flags=re.M)[1:]:
            name, rest = part.split(">:\n", 1)
            found[name] = Code(rest.splitlines())
    return found


def _code(*lines):
    """Instructions of four bytes each, jumps as the listing has them."""
    return Code([f"{line} // {0x4000 + 4 * i:012X}: 00000000" for i, line in enumerate(lines)])


def test_the_checks_see_what_they_are_for():
    use = "buffer_load_dwordx4 v1, s[4:7], s9 offen lds"
    # over a back edge: the descriptor is read back from lanes at the end of the loop and used at its beginning
    loop = _code(use, "v_add_u32_e32 v1, 1, v1", "v_readlane_b32 s4, v9, 1", "s_cmp_eq_u32 s1, s2", f"s_cbranch_scc0 {65536 - 5}", "s_endpgm")
    assert scalars_not_there_yet(loop) == [(2, 0)]
    assert not scalars_not_there_yet(_code("s_nop 4", use, "v_readlane_b32 s4, v9, 1", f"s_cbranch_scc0 {65536 - 4}", "s_endpgm"))
    # into either side of a branch, and not past its end
    assert scalars_not_there_yet(_code("v_readfirstlane_b32 s5, v0", "s_cbranch_scc1 1", "s_endpgm", use)) == [(0, 3)]
    assert not scalars_not_there_yet(_code("v_readfirstlane_b32 s5, v0", "s_branch 1", use, "s_endpgm"))
    # other writers of scalar registers
    assert scalars_not_there_yet(_code("v_add_co_u32_e64 v0, s[6:7], v1, v2", use))
    assert scalars_not_there_yet(_code("v_cmp_lt_u32_e64 s[4:5], v1, v2", "s_nop 3", use)) and not scalars_not_there_yet(_code("v_cmp_lt_u32_e64 s[4:5], v1, v2", "s_nop 4", use))
    assert scalars_not_there_yet(_code("v_cmp_lt_u32_e32 vcc, v1, v2", "global_load_dword v0, v1, vcc"))
    # data overwritten behind a jump, and in accumulators
    store = "buffer_store_dwordx4 v[42:45], v56, s[4:7], s88 offen"
    assert data_overwritten(_code("v_mov_b32_e32 v43, 0", store, f"s_branch {65536 - 3}")) == [(1, 0)]
    assert not data_overwritten(_code("v_mov_b32_e32 v43, 0", store, "s_nop 1", f"s_branch {65536 - 4}"))
    store = "buffer_store_dwordx4 a[0:3], v56, s[4:7], 0 offen"
    assert data_overwritten(_code(store, "v_accvgpr_write_b32 a2, v1")) and not data_overwritten(_code(store, "s_nop 1", "v_accvgpr_write_b32 a2, v1"))
    assert not data_overwritten(_code(store, "v_mov_b32_e32 v2, v1"))


def test_scalar_registers_are_there_on_every_way_to_a_memory_instruction(kernels):
    assert len(kernels) >= 300 and sum(len(c.ops) for c in kernels.values()) > 500000
    bad = {name: [(code.ops[i], code.ops[j]) for i, j in found[:2]] for name, code in kernels.items() if (found := scalars_not_there_yet(code))}
    assert not bad, bad


def test_data_of_wide_stores_stays_on_every_way_behind_them(kernels):
    bad = {name: [(code.ops[i], code.ops[j]) for i, j in found[:2]] for name, code in kernels.items() if (found := data_overwritten(code))}
    assert not bad, bad
