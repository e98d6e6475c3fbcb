"""Wait states around the matrix instructions of the tiles on 4-bit weights, read back from the built library (they are assembly that the
compiler does not know as such; see test_mfma_code_cpu, whose reader and rules these are)."""
import re
import shutil
import subprocess

import pytest

import test_mfma_code_cpu as code_check
from paper_2505_14468_amd.build import LIB_PATH

pytestmark = pytest.mark.skipif(not shutil.which(code_check.LLVM + "llvm-objdump"), reason="no disassembler")

VALU_TO_ADDRESS = 5  # a vector instruction that writes a scalar register, then a load that takes its descriptor or offset from it
SCALED_TO_ACCESS = 12  # a block-scaled 16x16x128 MFMA, then anything else that touches its accumulator


def _kernels(obj):
    text = subprocess.run([code_check.LLVM + "llvm-objdump", "-d", "--mcpu=gfx950", str(obj)], check=True, stdout=subprocess.PIPE, text=True).stdout
    for name, body in re.findall(r"^[0-9a-f]+ <(\S*mx_gemm_kernel\S*)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", text, re.S | re.M):
        code, base = [], None
        for line in body.splitlines():
            m = re.match(r"\s+(\S.*?)\s*// ([0-9A-F]+):", line)
            if not m or m[1].startswith("."):
                continue
            addr = int(m[2], 16)
            base = addr if base is None else base
            t = re.search(r"<\S+\+0x([0-9a-f]+)>", line) if "branch" in m[1] else None
            code.append(code_check.Instr(addr, m[1], base + int(t[1], 16) if t else (base if "branch" in m[1] else None)))
        yield name, code


def _scalars(text):
    return {i for a, b, c in re.findall(r"\bs(?:(\d+)|\[(\d+):(\d+)\])", text) for i in (range(int(b), int(c) + 1) if b else [int(a)])}


def stale_addresses(code):
    """Direct loads (assembly, so the compiler keeps no distance in front of them) that could read a scalar register too early."""
    prev = code_check.before(code)
    out = []
    for i, x in enumerate(code):
        if x.lds_load:
            for w in code_check.writers(code, prev, i, VALU_TO_ADDRESS):
                if w.valu and _scalars(w.text.split(",")[0]) & _scalars(x.text):
                    out.append((w.text, x.text))
    return out


def test_wait_states_of_every_tile(tmp_path):
    found = {}
    for k, data in enumerate(code_check.code_objects(LIB_PATH, tmp_path)):
        if b"mx_gemm_kernel" in data:
            obj = tmp_path / f"object_{k}"
            obj.write_bytes(data)
            found.update(_kernels(obj))
    assert len(found) == 14  # three tiles, one or two parts, whole or split; two of two tiles
    for name, code in found.items():
        scaled = [x for x in code if x.op.startswith("v_mfma_scale")]
        assert len(scaled) >= 64 and sum(x.lds_load for x in code) >= 6, name
        assert not code_check.faults(code), (name, code_check.faults(code)[:3])
        prev = code_check.before(code)
        since = code_check.states_since(code, prev, lambda x: x.op.startswith("v_mfma_scale"))
        accumulators = {r for x in scaled for r in x.dst}
        close = [(x.text, since[i]) for i, x in enumerate(code) if not x.mfma and x.regs & accumulators and since[i] < SCALED_TO_ACCESS]
        assert not close, (name, close[:3])
        assert not stale_addresses(code), (name, stale_addresses(code)[:3])


@pytest.mark.parametrize("code,found", [
    (["v_readfirstlane_b32 s4, v1", "s_nop 3", "buffer_load_dwordx4 v1, s[8:11], s4 offen lds", "s_endpgm"], True),
    (["v_readfirstlane_b32 s4, v1", "s_nop 4", "buffer_load_dwordx4 v1, s[8:11], s4 offen lds", "s_endpgm"], False),
    (["v_readlane_b32 s9, v1, 3", "s_add_i32 m0, s0, 16", "s_nop 0", "buffer_load_dwordx4 v1, s[8:11], s4 offen lds", "s_endpgm"], True),
    (["s_mov_b32 s9, s1", "buffer_load_dwordx4 v1, s[8:11], s4 offen lds", "s_endpgm"], False),
])
def test_the_check_finds_stale_addresses(code, found):
    assert bool(stale_addresses([code_check.Instr(4 * i, t, None) for i, t in enumerate(code)])) == found
