"""What the compiler made of the kernels of the layer norms and of attention, read off the built library."""

import re
import subprocess
import tempfile

import pytest

from tests import code_objects


@pytest.fixture
def kernels(monkeypatch):
    # mangled names: instances differ in types, which the short names leave out
    monkeypatch.setattr(code_objects, "short_name", str)
    return code_objects.kernel_metadata()


# instances: types x pieces x ways of a row's end; head sizes x workgroup sizes
@pytest.mark.parametrize("name,instances", [("layer_norm_kernel", 48), ("layer_norm_backward_kernel", 48), ("layer_norm_sum_kernel", 1),
                                            ("attention_kernel", 8), ("attention_few_kernel", 4), ("attention_join_kernel", 4),
                                            ("attention_row_grad_kernel", 4), ("attention_key_grad_kernel", 4), ("attention_grad_join_kernel", 4)])
def test_rows_and_sums_stay_in_registers(kernels, name, instances):
    mine = {n: k for n, k in kernels.items() if re.search(rf"\d{name}[EI]", n)}
    assert len(mine) == instances
    for n, k in mine.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, f"{n} spills"


# two workgroups of four waves to a compute unit, one of eight: two waves to a SIMD of 512 registers
@pytest.mark.parametrize("name", ["attention_kernel", "attention_row_grad_kernel", "attention_key_grad_kernel"])
def test_two_waves_fit_a_simd(kernels, name):
    for n, k in kernels.items():
        if re.search(rf"\d{name}I", n):
            assert k[".vgpr_count"] + k.get(".agpr_count", 0) <= 256, n


def _code(names):
    """{kernel: its instructions as (mnemonic, operands, place of the branch's target or None)} of kernels whose names match."""
    out = {}
    for elf in code_objects.code_objects():
        with tempfile.NamedTemporaryFile(suffix=".elf") as f:
            f.write(elf)
            f.flush()
            text = subprocess.run([code_objects.OBJDUMP, "-d", "--mcpu=gfx950", "--no-show-raw-insn", f.name], check=True, capture_output=True,
                                  text=True).stdout
        body = None
        for line in text.splitlines():
            label = re.match(r"([0-9a-f]+) <(\S+)>:", line)
            if label:
                body = out.setdefault(label[2], (int(label[1], 16), [])) if re.search(names, label[2]) else None
            elif body and line.startswith("\t"):
                code, _, rest = line.partition("//")
                name, _, operands = code.strip().partition(" ")
                if not rest:        # padding behind the code
                    continue
                target = re.search(r"<\S+?(?:\+0x([0-9a-f]+))?>", rest) if "branch" in name else None
                body[1].append((int(rest.split(":")[0], 16) - body[0], name, operands.strip(), int(target[1] or "0", 16) if target else None))
    return {n: _placed(code) for n, (_, code) in out.items()}


def _placed(code):
    """Addresses of branches' targets as places in the code."""
    place = {at: i for i, (at, *_) in enumerate(code)}
    return [(name, operands, None if to is None else place[to]) for _, name, operands, to in code]


def _loads_beside_reads(code):
    """The places of loads into LDS that a read of LDS may reach along some way without a wait for all of them between."""
    found, seen, todo = set(), set(), [(0, False)]
    while todo:
        at, reads = todo.pop()
        if (at, reads) in seen or at >= len(code):
            continue
        seen.add((at, reads))
        name, operands, to = code[at]
        if name.startswith("ds_read"):
            reads = True
        elif name == "s_waitcnt" and ("lgkmcnt(0)" in operands or operands.strip() == "0"):
            reads = False
        elif "load_lds" in name and reads:
            found.add(at)
        if to is not None:
            todo.append((to, reads))
        if name not in ("s_branch", "s_endpgm", "s_setpc_b64"):
            todo.append((at + 1, reads))
    return sorted(found)


def test_loads_beside_reads_are_seen():
    read, load, wait = ("ds_read_b128", "v[0:3], v4", None), ("global_load_lds_dwordx4", "v2, s[4:5]", None), ("s_waitcnt", "lgkmcnt(0)", None)
    some, again, end = ("s_waitcnt", "vmcnt(0) lgkmcnt(3)", None), ("s_cbranch_vccnz", "65533", 0), ("s_endpgm", "", None)
    assert _loads_beside_reads([load, read, wait, again, end]) == []
    assert _loads_beside_reads([load, read, some, again, end]) == [0]      # round the loop
    assert _loads_beside_reads([read, ("s_branch", "1", 3), wait, load, end]) == [3]
    assert _loads_beside_reads([read, wait, load, end]) == [] and _loads_beside_reads([read, end, load]) == []


def test_tiles_are_loaded_over_ones_that_have_been_read():
    # a load into LDS begins when the reads before it have arrived: of the tile that it replaces, among them
    kernels = _code(r"\d+attention_(few_|row_grad_|key_grad_)?kernelI")
    assert len(kernels) == 20
    for n, code in kernels.items():
        assert any("load_lds" in i[0] for i in code) and any(i[0].startswith("ds_read") for i in code), n
        assert _loads_beside_reads(code) == [], n


def test_waits_for_reads_are_in_the_source():
    # a wave of few rows refills a buffer that it alone has read, without a barrier
    with open(code_objects.oq.__path__[0] + "/csrc/attention.hip") as f:
        few = re.search(r"void attention_few_kernel.*?\n}\n", f.read(), re.S)[0]
    loop = few[few.index("for (int buffer"):]
    assert re.search(r"reads_done\(\);\s*load\(", loop) and loop.count(" load(") == 1


def _strays_of_m0(code):
    """The places where m0 is used otherwise than by a move to it, a wait state and the load into LDS that takes it."""
    found = []
    for at, (name, operands, _) in enumerate(code):
        words = re.split(r"[ ,\[\]:]+", operands)
        if "load_lds" in name:
            before = [i[:2] for i in code[max(0, at - 2):at]]
            ok = len(before) == 2 and before[0][0] == "s_mov_b32" and before[0][1].startswith("m0,") and before[1] == ("s_nop", "0")
        elif name == "s_mov_b32" and words[0] == "m0":
            ok = at + 2 < len(code) and "load_lds" in code[at + 2][0]
        else:   # instructions that name it, or take it unsaid: moves indexed by it, messages
            ok = "m0" not in words and not name.startswith(("v_movrel", "s_movrel", "s_sendmsg", "ds_gws", "ds_ordered"))
        if not ok:
            found.append(at)
    return found


def test_strays_of_m0_are_seen():
    move, wait, load = ("s_mov_b32", "m0, s4", None), ("s_nop", "0", None), ("global_load_lds_dwordx4", "v2, s[4:5]", None)
    assert _strays_of_m0([move, wait, load, move, wait, load]) == []
    assert _strays_of_m0([move, wait, load, wait, load]) == [4] and _strays_of_m0([move, load]) == [0, 1]
    assert _strays_of_m0([("v_readlane_b32", "s3, v1, m0", None)]) == [0] and _strays_of_m0([("v_movrels_b32_e32", "v1, v2", None)]) == [0]


def test_loads_into_lds_have_m0_to_themselves():
    # the inline assembly that writes m0 does not say so: the compiler reserves the register, warns of its name in a list of
    # clobbers, and must keep nothing of its own in it across a load
    kernels = _code(r"\d+attention_(few_|row_grad_|key_grad_)?kernelI")
    assert len(kernels) == 20
    for n, code in kernels.items():
        assert any("load_lds" in i[0] for i in code) and _strays_of_m0(code) == [], n
