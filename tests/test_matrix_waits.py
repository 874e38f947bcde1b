"""Issue slots between a bf16 matrix product and what touches its registers, in the built kernels.  The hardware does not wait for these
by itself; the compiler puts idle slots where it sees who reads, and does not see into inline assembly.  Read from the disassembly of the
library's own code objects, along every path through the branches; no GPU needed."""
import os
import re
import struct
import subprocess

import pytest

import paper_2604_10103_amd as hf

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
PASSES = {"v_mfma_f32_32x32x16_bf16": 8}   # of four cycles each
REGISTERS = re.compile(r"\b([va])(?:(\d+)|\[(\d+):(\d+)\])")
INSTRUCTION = re.compile(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]+):(.*)")
READERS = ("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")


def _registers(text):
    found = set()
    for kind, one, lo, hi in REGISTERS.findall(text):
        found.update((kind, r) for r in range(int(one or lo), int(one or hi) + 1))
    return frozenset(found)


def _operands(text):
    return [_registers(x) for x in re.split(r",(?![^\[]*\])", text)]


def _code_objects():
    with open(os.path.join(os.path.dirname(hf.__file__), "libhf.so"), "rb") as f:
        lib = f.read()
    at = lib.find(b"__CLANG_OFFLOAD_BUNDLE__")
    while at >= 0:
        n, = struct.unpack_from("<Q", lib, at + 24)
        p = at + 32
        for _ in range(n):
            off, size, triple = struct.unpack_from("<QQQ", lib, p)
            if size and b"gfx950" in lib[p + 24:p + 24 + triple]:
                yield lib[at + off:at + off + size]
            p += 24 + triple
        at = lib.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 24)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Mangled name -> [(opcode, operands as text, address, rest of the line)]"""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump here")
    found = {}
    for i, code in enumerate(_code_objects()):
        path = tmp_path_factory.mktemp("code") / f"{i}.co"
        path.write_bytes(code)
        name = None
        for line in subprocess.run([OBJDUMP, "-d", str(path)], capture_output=True, text=True, check=True).stdout.split("\n"):
            label = re.match(r"^[0-9a-f]+ <(.*)>:", line)
            if label:
                name = label[1]
                found[name] = []
            elif name:
                m = INSTRUCTION.match(line)
                if m:
                    found[name].append((m[1], m[2], int(m[3], 16), m[4]))
    return found


def too_early(code):
    """(what, product's address, reader's address, slots between, slots needed) of every access that comes too early."""
    index = {x[2]: i for i, x in enumerate(code)}
    operands = {}

    def ops(i):
        if i not in operands:
            operands[i] = _operands(code[i][1]) if code[i][0].startswith(READERS) else []
        return operands[i]

    def after(i):
        op, _, _, rest = code[i]
        to = []
        if op.startswith(("s_cbranch", "s_branch")):
            to.append(index[code[0][2] + int(re.search(r"\+0x([0-9a-f]+)>", rest)[1], 16)])
        if op not in ("s_branch", "s_endpgm") and i + 1 < len(code):
            to.append(i + 1)
        return to

    def reach(i, most, live):
        """Instructions within `most` slots behind i, with the slots between and what of `live` no later product has written since."""
        seen, open_ = {}, [(j, 0, live) for j in after(i)]
        while open_:
            j, slots, regs = open_.pop()
            if slots >= most or not regs or seen.get((j, regs), most) <= slots:
                continue
            seen[j, regs] = slots
            yield j, slots, regs
            if code[j][0] in PASSES:
                regs = regs - ops(j)[0]
            slots += int(code[j][1], 0) + 1 if code[j][0] == "s_nop" else 1
            open_ += [(k, slots, regs) for k in after(j)]

    found = []
    for i, (op, _, address, _) in enumerate(code):
        if op not in PASSES:
            continue
        result, _, _, start = ops(i)[:4]
        written = PASSES[op] + 4
        for j, slots, live in reach(i, written, result):
            mine = ops(j)
            if code[j][0] in PASSES:   # (its third operand may be the result: products that add up follow each other)
                touches = (mine[1] | mine[2]) & live
            else:
                touches = any(x & live for x in mine)
            if touches:
                found.append(("reads or overwrites the result", hex(address), hex(code[j][2]), slots, written))
        if start and start != result:
            for j, slots, _ in reach(i, PASSES[op] - 1, result | start):
                if code[j][0].startswith("v_") and code[j][0] not in PASSES and ops(j)[0] & start:
                    found.append(("overwrites what the product starts from", hex(address), hex(code[j][2]), slots, PASSES[op] - 1))
    return found


def test_the_search_itself():
    def program(*lines):
        return [(x.split(" ", 1)[0], x.split(" ", 1)[1] if " " in x else "", 4 * i, "") for i, x in enumerate(lines)]
    product = "v_mfma_f32_32x32x16_bf16 v[0:15], v[20:23], v[24:27], v[0:15]"
    assert [x[3:] for x in too_early(program(product, "s_nop 3", "s_add_u32 s0, s0, s1", "v_max3_f32 v30, v3, v4, v31"))] == [(5, 12)]
    assert not too_early(program(product, "s_nop 11", "v_max3_f32 v30, v3, v4, v31"))
    assert not too_early(program(product, "v_add_f32_e32 v30, v16, v31", product))
    assert too_early(program(product, "v_mfma_f32_32x32x16_bf16 v[40:55], v[12:15], v[24:27], v[40:55]"))
    from_other = "v_mfma_f32_32x32x16_bf16 a[0:15], v[20:23], v[24:27], v[0:15]"
    assert [x[3:] for x in too_early(program(from_other, "s_nop 0", "v_mul_f32_e32 v2, v30, v31"))] == [(1, 7)]
    assert not too_early(program(from_other, "s_nop 6", "v_mul_f32_e32 v2, v30, v31"))
    jump = program(product, "s_cbranch_scc1 4", "s_nop 15", "s_endpgm", "v_mov_b32_e32 v30, v15")
    jump[1] = jump[1][:3] + (" <x+0x10>",)
    assert [x[1:4] for x in too_early(jump)] == [("0x0", "0x10", 1)]


@pytest.mark.parametrize("family", ["paged_attn_kernel", "attn_mfma_kernel", "attn_d64_kernel", "attn_split_kernel", "attn_w64_kernel", "bwd_mfma_kernel",
                                    "absorb_quad_kernel", "absorb_mfma_kernel", "readout_mfma_kernel"])
def test_results_of_products_are_waited_for(kernels, family):
    some = {n: code for n, code in kernels.items() if family in n and any(x[0] in PASSES for x in code)}
    assert some
    assert {n: bad for n, bad in ((n, too_early(code)) for n, code in some.items()) if bad} == {}
