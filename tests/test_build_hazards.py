"""The built kernels have the wait states that the hardware leaves to the program, also where the compiler does not see to them: it looks neither into
inline assembly nor at what stands in front of it.  Read from the library's own code, instruction by instruction in the order of their addresses:

  a vector instruction writes a scalar register, a memory instruction reads it       5 wait states
  a vector instruction writes a register, a matrix instruction reads it              2
  a matrix instruction (16 x 16, 8 passes) writes a register, another one touches it 11

An instruction is a wait state, s_nop n is n + 1."""
import os
import re
import subprocess

import pytest

import paper_2401_08383_amd as exf

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
REGISTERS = re.compile(r"([vas])(?:\[(\d+):(\d+)\]|(\d+))$")
# kernels whose matrix instructions are inline assembly
ASSEMBLY = re.compile(r"grouped_gemm|rows_tiles_kernel|weight_tiles_kernel|weight_stream_kernel")
CARRIES = ("v_add_co", "v_sub_co", "v_subrev_co", "v_addc_co", "v_subb_co", "v_div_scale", "v_mad_u64", "v_mad_i64")  # (their second result is a scalar pair)


def _registers(token):
    m = REGISTERS.match(token.strip("-|"))
    if not m:
        return frozenset()
    first, last = (int(m[2]), int(m[3])) if m[2] else (int(m[4]), int(m[4]))
    return frozenset((m[1], i) for i in range(first, last + 1))


def hazards(lines):
    """(kind, kernel, earlier instruction, later one) of every pair that is too close."""
    found, kernel, recent, products = [], "", [], []
    for line in lines:
        text = line.split("//")[0].strip()
        if not text:
            continue
        if text.endswith(">:"):
            kernel, recent, products = text[1:-2], [], []
            continue
        op, _, rest = text.partition(" ")
        tokens = [t.strip().split(" ")[0] for t in rest.split(",")] if rest else []
        states = int(tokens[0], 0) + 1 if op == "s_nop" else 1
        matrix, memory = op.startswith("v_mfma"), op.startswith(("buffer_", "global_", "flat_", "scratch_"))

        def look_back(need, read, kind):
            past = 0
            for earlier, written, length in reversed(recent):
                if past >= need:
                    return
                if written & read:
                    found.append((kind, kernel, earlier, text))
                    return
                past += length

        if matrix:
            look_back(2, frozenset().union(*map(_registers, tokens[1:])), "vector result, matrix operand")
        if memory:
            look_back(5, frozenset(r for t in tokens for r in _registers(t) if r[0] == "s"), "scalar of a vector instruction, memory operand")
        touched = frozenset().union(*map(_registers, tokens)) if tokens and not matrix and op != "s_nop" else frozenset()
        for product in products:
            if product[1] < 11 and product[0] & touched:
                found.append(("matrix result, other instruction", kernel, product[2], text))
                break
        written = frozenset()
        if op.startswith("v_") and not matrix and tokens:
            written = _registers(tokens[0]) | (_registers(tokens[1]) if op.startswith(CARRIES) else frozenset())
        if matrix and ASSEMBLY.search(kernel):
            products = [p for p in products if p[1] < 11] + [[_registers(tokens[0]), 0, text]]
        for product in products:
            product[1] += states
        recent = recent[-6:] + [(text, written, states)]
    return found


def test_the_scan_sees_what_is_too_close():
    """... on listings of a few lines."""
    def of(*lines):
        return [h[0] for h in hazards(["<rows_tiles_kernel>:", *lines])]

    read = "global_load_lds_dword v2, s[26:27]"
    assert of("v_readlane_b32 s27, v80, 1", "s_mov_b32 m0, s3", "s_nop 0", read) == ["scalar of a vector instruction, memory operand"]
    assert of("v_readlane_b32 s27, v80, 1", "s_mov_b32 m0, s3", "s_nop 3", read) == []
    assert of("v_readfirstlane_b32 s25, v80", read) == []
    multiply = "v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]"
    assert of("v_mov_b32_e32 v5, 0", multiply) == ["vector result, matrix operand"] == of("v_mov_b32_e32 v11, 0", "s_nop 0", multiply)
    assert of("v_mov_b32_e32 v5, 0", "s_nop 1", multiply) == []
    assert of(multiply, "s_nop 8", "v_accvgpr_read_b32 v1, a2") == ["matrix result, other instruction"]
    assert of(multiply, "s_nop 9", "v_accvgpr_read_b32 v1, a2") == [] == of(multiply, multiply)


def test_wait_states(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("needs the toolchain's llvm-objdump")
    exf.lib()
    library = tmp_path / "lib.so"
    library.symlink_to(exf.LIB_PATH)
    subprocess.run([OBJDUMP, "--offloading", str(library)], cwd=tmp_path, check=True, capture_output=True)
    images = sorted(p for p in tmp_path.iterdir() if p.name.endswith("gfx950"))
    assert len(images) > 10
    found = []
    for image in images:
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(image)], check=True, capture_output=True, text=True).stdout
        assert "s_endpgm" in listing
        found += hazards(listing.splitlines())
    assert not found, f"{len(found)} pairs too close, the first: {found[:3]}"
