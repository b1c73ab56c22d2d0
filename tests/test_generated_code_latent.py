"""Checks on the machine code hipcc generates for the operators on a latent cache and for rows from logits (no GPU needed: they are
only compiled).  Properties that their correctness or speed depend on and that another compiler could silently take away."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2409_10644_amd.build import COMMON, CSRC, SOURCES

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FILES = ("tree_attention_latent.hip", "latent_rows.hip", "sample_rows.hip")


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    """{mangled kernel name: lines of code}, {kernel name: {resource: number}}"""
    if not (os.path.exists(HIPCC) or shutil.which(HIPCC)):
        pytest.skip("hipcc not available")
    code, numbers = {}, {}
    for name in FILES:
        out = tmp_path_factory.mktemp("asm") / "out.s"
        subprocess.run([HIPCC, *COMMON, *SOURCES[name], "-S", "--cuda-device-only", "-o", str(out), os.path.join(CSRC, name)], check=True, capture_output=True)
        body = last = None
        for l in out.read_text().split("\n"):
            m = re.match(r"^(_Z\w+kernel\w*):", l)
            if m:
                last = m.group(1)
                body = code.setdefault(last, [])
            elif l.startswith(".Lfunc_end"):
                body = None
            elif body is not None:
                if l.split(";")[0].strip():
                    body.append(l.split(";")[0].strip())
            m = re.match(r"^; (ScratchSize|NumVgprs|VGPR Blocks|Occupancy): (\d+)", l)
            if m and last:
                numbers.setdefault(last, {})[m.group(1)] = int(m.group(2))
    return code, numbers


def _sweeps(code):
    return {n: b for n, b in code.items() if "tree_attn_latent_kernel" in n}


def test_every_variant_is_there(listings):
    found = sorted(re.search(r"latent_kernelILi(\d+)ELi(\d+)ELb(\d)E", n).groups() for n in _sweeps(listings[0]))
    assert found == [("256", "32", "0"), ("256", "32", "1"), ("512", "64", "0"), ("512", "64", "1")]
    assert sum("sample_rows_kernel" in n for n in listings[0]) == 4


def test_what_a_lane_holds_stays_in_registers(listings):
    """The queries and the output of the attention, and the rows' numbers, without a trip to memory; two wavefronts of 256 registers to a
    SIMD.  (The sampling kernel trades a few of its own for a second workgroup.)"""
    assert set(listings[1]) == set(listings[0]) and all("ScratchSize" in n for n in listings[1].values())
    for name, n in listings[1].items():
        if "sample_rows" not in name:
            assert n["ScratchSize"] == 0, (name, n)
            assert not any(l.startswith("scratch_") for l in listings[0][name]), name
        else:
            assert n["ScratchSize"] <= 128, (name, n)


def test_no_packed_fp32(listings):
    for name, body in listings[0].items():
        assert not any(re.match(r"v_pk_(add|mul|fma)_f32", l) for l in body), name


def _vectors(text):
    found = set()
    for a, b in re.findall(r"\bv\[(\d+):(\d+)\]", text):
        found |= set(range(int(a), int(b) + 1))
    return found | {int(a) for a in re.findall(r"\bv(\d+)\b", text)}


def test_products_are_done_before_vector_instructions_touch_them(listings):
    """The matrix instructions are the source's own, so the wait states behind them are too: 11 between a product of 8 passes and another
    instruction at its registers (an accumulation into the same ones needs none)."""
    for name, body in _sweeps(listings[0]).items():
        states, written, products = 0, {}, 0
        for l in body:
            if l.startswith(".") or l.endswith(":"):
                continue
            if l.startswith("s_nop"):
                states += int(l.split()[1], 0) + 1
                continue
            operands = l.split(None, 1)[1] if " " in l or "\t" in l else ""
            if l.startswith("v_mfma"):
                dst, a, b, c = [x.strip() for x in operands.split(", ")]
                assert dst == c, (name, l)
                touched = _vectors(a) | _vectors(b)
                products += 1
            else:
                touched = _vectors(operands)
            close = [r for r in touched if r in written and states - written[r] < 11]
            assert not close, (name, l, close)
            states += 1
            if l.startswith("v_mfma"):
                written.update((r, states) for r in _vectors(dst))
            elif l.startswith("v_"):
                for r in _vectors(operands.split(",")[0]):
                    written.pop(r, None)
        assert products >= 16 + 36 or "Li256ELi32" in name and products >= 16 + 18, (name, products)


def test_vector_instructions_are_done_before_products_read_them(listings):
    """Two wait states between a vector instruction's result and a matrix instruction that reads it, on the way through the code in its
    order and from every branch back to its target (results of loads are waited for by the compiler)."""
    for name, body in _sweeps(listings[0]).items():
        labels = {l[:-1]: i for i, l in enumerate(body) if l.endswith(":")}
        ways = [range(len(body))]
        for i, l in enumerate(body):
            m = re.match(r"s_c?branch\w*\s+(\.L\w+)", l)
            if m and m.group(1) in labels:
                at = labels[m.group(1)]
                ways.append([*range(max(0, i - 4), i + 1), *range(at, min(at + 4, len(body)))])
        for way in ways:
            states, written = 0, {}
            for i in way:
                l = body[i]
                if l.startswith(".") or l.endswith(":"):
                    continue
                if l.startswith("s_nop"):
                    states += int(l.split()[1], 0) + 1
                    continue
                operands = l.split(None, 1)[1] if len(l.split(None, 1)) > 1 else ""
                if l.startswith("v_mfma"):
                    close = [r for r in _vectors(operands) if r in written and states - written[r] < 2]
                    assert not close, (name, l, close)
                states += 1
                if l.startswith("v_mfma"):
                    for r in _vectors(operands.split(",")[0]):
                        written.pop(r, None)
                elif l.startswith("v_"):
                    written.update((r, states) for r in _vectors(operands.split(",")[0]))


def test_the_variant_for_few_rows(listings):
    """Both sizes are there, with as many products as their rows need, and its wait states are those of the others."""
    few = {n: b for n, b in listings[0].items() if "tree_attn_latent_few_kernel" in n}
    assert sorted(re.search(r"few_kernelILi(\d+)ELi(\d+)E", n).groups() for n in few) == [("256", "32"), ("512", "64")]
    renamed = {n.replace("latent_few_kernel", "latent_kernel"): b for n, b in few.items()}
    test_vector_instructions_are_done_before_products_read_them((renamed, {}))
    for name, body in few.items():
        products = [i for i, l in enumerate(body) if l.startswith("v_mfma")]
        assert len(products) >= (18 + 8 if "Li512" in name else 9 + 4), name
        for i in products:                                     # what a product writes, no other instruction touches within 11 wait states
            written, states = _vectors(body[i].split(None, 1)[1].split(",")[0]), 0
            for l in body[i + 1:]:
                if l.startswith(".") or l.endswith(":"):
                    continue
                if l.startswith("s_nop"):
                    states += int(l.split()[1], 0) + 1
                    continue
                if states >= 11 or l.startswith("s_cbranch") or l.startswith("s_branch"):
                    break
                operands = l.split(None, 1)[1] if len(l.split(None, 1)) > 1 else ""
                if l.startswith("v_mfma"):
                    operands = ", ".join(operands.split(", ")[1:3])
                assert not written & _vectors(operands), (name, body[i], l)
                states += 1
