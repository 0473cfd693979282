"""Results of matrix instructions are not there at once, and nothing in the hardware holds back who reads them too early: the
compiler counts instructions and fills up with s_nop.  On the taken way of a branch it has left too few once, which gave
wrong scores.  So every way through every kernel that was built is walked here, from each matrix instruction to the
first use of its result."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_09844_amd import SO

# Wait states from an instruction to a use of its result: its passes of 4 cycles and 4 more (bf16: 4 and 8 passes), or 2 more
# (fp32: 8 and 16), as the compiler leaves them in straight code.
NEEDED = {"16x16x32_bf16": 8, "32x32x16_bf16": 12, "16x16x4_f32": 10, "32x32x2_f32": 18}
OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")


def registers(text):
    """Vector and accumulation registers that operands name."""
    out = set()
    for kind, lo, hi, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out |= {(kind, i) for i in (range(int(lo), int(hi) + 1) if lo else (int(one),))}
    return out


def parse(listing):
    """Kernels of a disassembly: name -> list of (mnemonic, operands, target's index or None)."""
    kernels, rows = {}, None
    for line in listing.splitlines():
        m = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
        if m:
            rows = kernels.setdefault(m[1], [])
            continue
        m = re.match(r"^\s+([a-z]\S*)\s*(.*?)\s*// ([0-9A-F]+): ", line)
        if m and rows is not None:
            rows.append((m[1], m[2], int(m[3], 16)))
    for name, rows in kernels.items():
        index = {at: i for i, (_, _, at) in enumerate(rows)}
        for i, (op, args, at) in enumerate(rows):
            target = None
            if op.startswith(("s_branch", "s_cbranch")):
                jump = int(args.split()[0])
                target = index[at + 4 + 4 * (jump - (1 << 16) if jump >= 1 << 15 else jump)]
            rows[i] = (op, args, target)
    return kernels


def early(rows):
    """Uses of results that come too early: (matrix instruction, use, wait states between)."""
    found = []
    uses = [registers(args) for _, args, _ in rows]
    for i, (op, args, _) in enumerate(rows):
        if not op.startswith("v_mfma_"):
            continue
        need = NEEDED[re.match(r"v_mfma_f32_(\w+?)(?:_e64)?$", op)[1]]
        result = registers(args.split(",")[0] if "[" not in args.split(",")[0] else args[: args.index("]") + 1])
        ways, least = [(i + 1, 0)], {}
        while ways:
            k, states = ways.pop()
            if k >= len(rows) or states >= need or least.get(k, need) <= states:
                continue
            least[k] = states
            op2, args2, target = rows[k]
            if op2.startswith("v_mfma_"):
                parts = re.split(r",\s*(?![^\[]*\])", args2)
                if (registers(parts[1]) | registers(parts[2])) & result:
                    found.append((f"{op} {args}", f"{op2} {args2}", states))
                    continue
                if registers(parts[0]) & result:  # (as the addend of the next one it is passed on)
                    continue
            elif op2.startswith(("v_", "ds_", "buffer_", "global_", "flat_", "scratch_")) and uses[k] & result:
                found.append((f"{op} {args}", f"{op2} {args2}", states))
                continue
            if target is not None:
                ways.append((target, states + 1))
            if op2 not in ("s_branch", "s_endpgm"):
                ways.append((k + 1, states + (int(args2, 0) + 1 if op2 == "s_nop" else 1)))
    return found


def listing(*lines):
    return "0000000000000100 <k>:\n" + "".join(f"\t{x}    // {0x100 + 4 * i:012X}: 00000000 \n" for i, x in enumerate(lines))


MFMA = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]"


@pytest.mark.parametrize("lines,states", [
    ([MFMA, "s_nop 7", "v_mul_f32_e32 v9, v3, v4", "s_endpgm"], []),
    ([MFMA, "s_nop 6", "v_mul_f32_e32 v9, v3, v4", "s_endpgm"], [7]),
    ([MFMA, "s_cbranch_scc1 1", "s_nop 7", "s_nop 1", "v_add_f32_e32 v9, v3, v4", "s_endpgm"], [3]),  # the way without the s_nop 7
    ([MFMA, "s_cbranch_scc1 1", "s_nop 7", "s_nop 5", "v_add_f32_e32 v9, v3, v4", "s_endpgm"], [7]),
    (["v_add_f32_e32 v9, v3, v4", MFMA, "s_cbranch_scc1 65533", "s_endpgm"], [1]),  # back to the start
    ([MFMA, MFMA, "s_nop 7", "global_store_dword v[20:21], v2, off", "s_endpgm"], []),
    ([MFMA, "v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[12:15], v[4:7]", "s_nop 7", "s_endpgm"], [0]),
    ([MFMA, "s_branch 1", "ds_write_b32 v30, v1", "v_mov_b32_e32 v31, v16", "s_endpgm"], []),
], ids=range(8))
def test_the_walk_finds_uses_that_come_too_early(lines, states):
    assert [s for _, _, s in early(parse(listing(*lines))["k"])] == states


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    path = tmp_path_factory.mktemp("code")
    so = shutil.copy(SO, path / "lib.so")
    subprocess.check_call([OBJDUMP, "--offloading", str(so)], cwd=path, stdout=subprocess.DEVNULL)
    out = {}
    for f in sorted(path.iterdir()):
        if "amdgcn" in f.name:
            out.update({(f.name, n): r for n, r in parse(subprocess.check_output([OBJDUMP, "-d", str(f)], text=True)).items()})
    return out


def test_no_result_of_a_matrix_instruction_is_used_too_early(kernels):
    matrix = {k: r for k, r in kernels.items() if any(op.startswith("v_mfma_") for op, _, _ in r)}
    for kernel in ("k_pdecode", "k_pprompt_bf16", "k_pprompt_f32", "k_pprompt_split"):
        assert any(kernel in name for _, name in matrix), kernel
    bad = {name: found for (_, name), r in matrix.items() if (found := early(r))}
    assert not bad, "\n".join(f"{n}: {f[0][0]} -> {f[0][1]}, {f[0][2]} wait states" for n, f in bad.items())
