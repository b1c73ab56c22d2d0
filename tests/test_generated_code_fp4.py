"""Checks on the machine code hipcc generates for the attention over the 4-bit cache (no GPU needed: it is only compiled).
Properties that its correctness or its speed depend on and that another compiler could silently take away."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2409_10644_amd.build import COMMON, CSRC, SOURCES

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
KERNEL = re.compile(r"tree_attn_fp4_kernelILi(\d+)ELi(\d+)ELb(\d)E")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{(head_dim, query blocks, non-temporal): [(line of code, inside the source's own assembly)]}"""
    if not (os.path.exists(HIPCC) or shutil.which(HIPCC)):
        pytest.skip("hipcc not available")
    out = tmp_path_factory.mktemp("asm") / "fp4.s"
    subprocess.run([HIPCC, *COMMON, *SOURCES["tree_attention_fp4.hip"], "-S", "--cuda-device-only", "-o", str(out),
                    os.path.join(CSRC, "tree_attention_fp4.hip")], check=True, capture_output=True)
    found, body, inside = {}, None, False
    for l in out.read_text().split("\n"):
        if re.match(r"^_Z\w+:", l):
            m = KERNEL.search(l)
            body = found.setdefault(tuple(int(x) for x in m.groups()), []) if m else None
        elif l.startswith(".Lfunc_end"):
            body = None
        elif body is not None:
            if "#ASMSTART" in l or "#ASMEND" in l:
                inside = "#ASMSTART" in l
            elif l.split(";")[0].strip():
                body.append((l.split(";")[0].strip(), inside))
    return found


def _blocks(body):
    blocks, cur = [], []
    for l, _ in body:
        if re.match(r"^\.LBB\w+:", l):
            blocks.append(cur)
            cur = []
        cur.append(l)
    return blocks + [cur]


def _registers(operand):
    m = re.fullmatch(r"v\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m.group(1)), int(m.group(2)) + 1))
    m = re.fullmatch(r"v(\d+)", operand)
    return {int(m.group(1))} if m else set()


def test_every_variant_is_there(kernels):
    assert sorted(kernels) == sorted([(d, q, 1) for d in (64, 128) for q in (1, 2, 4)] + [(d, 4, 0) for d in (64, 128)])


def test_m0_is_only_touched_by_the_kernels_own_assembly(kernels):
    for name, body in kernels.items():
        uses = [(l, inside) for l, inside in body if re.search(r"\bm0\b", l)]
        assert uses and all(inside for _, inside in uses), name


def test_conversions_to_six_bits_do_not_overwrite_what_they_read(kernels):
    """They write first results while they still read: a destination on an operand gave wrong numbers."""
    for name, body in kernels.items():
        seen = 0
        for l, _ in body:
            m = re.match(r"v_cvt_scalef32_(?:2xpk16|pk32)\S*\s+(.*)", l)
            if m:
                ops = [o.strip() for o in m.group(1).split(",")]
                into = _registers(ops[0])
                assert into and not any(into & _registers(o) for o in ops[1:]), f"{name}: {l}"
                seen += 1
        assert seen == 5 * name[0] // 64, (name, seen)         # three terms, two of them read back


def test_the_steady_blocks_hold_everything_in_registers(kernels):
    """A block of 32 keys in the pipelined variants: scores, weights and products in one piece of code, nothing from or to memory but
    LDS, no copies of accumulators, no wait on vector memory, and most weights made between matrix instructions."""
    for name, body in kernels.items():
        if name[1] == 1:
            continue
        mfma = {128: 14, 64: 7}[name[0]]
        steady = [b for b in _blocks(body) if sum("v_mfma" in l for l in b) == mfma and sum("v_exp_f32" in l for l in b) == 16]
        assert len(steady) >= 2, name
        for b in steady:
            assert not any(re.search(r"scratch_|buffer_|global_", l) for l in b if "_lds_" not in l), name
            first = next(i for i, l in enumerate(b) if "v_mfma" in l)
            last = max(i for i, l in enumerate(b) if "v_mfma" in l)
            assert not any("vmcnt" in l for l in b[:last]), name
            assert sum(bool(re.match(r"v_mov_b(32|64)", l)) for l in b) <= 4, name
            assert sum("v_exp_f32" in l for l in b[first:last]) >= 12, name
            assert not any("v_dot2" in l for l in b), name      # (these occupy the matrix unit)


def test_the_steady_loops_spill_nothing(kernels):
    """From the first to the last of those blocks, and what stands between them: no register kept in memory."""
    for name, body in kernels.items():
        if name[1] == 1:
            continue
        mfma = {128: 14, 64: 7}[name[0]]
        blocks = _blocks(body)
        steady = [i for i, b in enumerate(blocks) if sum("v_mfma" in l for l in b) == mfma and sum("v_exp_f32" in l for l in b) == 16]
        assert not any("scratch_" in l for b in blocks[steady[0]:steady[-1] + 1] for l in b), name


def test_the_exchange_of_partial_results_needs_no_loops_over_descriptors(kernels):
    """A buffer descriptor that the compiler does not know to be uniform is read lane by lane, in a loop of a few instructions."""
    for name, body in kernels.items():
        code = [l for l, _ in body]
        at = {m.group(1): i for i, l in enumerate(code) if (m := re.match(r"^(\.LBB\w+):", l))}
        for i, l in enumerate(code):
            m = re.match(r"s_cbranch_execnz\s+(\.LBB\w+)", l)
            if m and 0 < i - at.get(m.group(1), i) < 40:
                assert not any("v_readfirstlane" in x for x in code[at[m.group(1)]:i]), name
