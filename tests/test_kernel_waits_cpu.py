"""Loads straight to LDS are waited for before the barrier behind which other waves read them, in the
compiler's own output for gfx950 (no GPU needed).

A barrier orders the waves' LDS instructions, but not such a load: the wave that started it has to
wait (vmcnt(0)) itself.  Without that the load is nearly always there in time, so that a run shows
nothing."""
import os
import re
import subprocess

import pytest

from paper_2606_24467_amd import build as B

LOAD = re.compile(r"\s+(global_load_lds_\w+|buffer_load_\w+\s.*\blds\b)")
BRANCH = re.compile(r"\s+(s_c?branch\S*)\s+(\.L\w+)")


def blocks_of(body):
    """A function's instructions as {label: (lines, labels of the next blocks)}."""
    blocks, label, lines, ends = {}, "entry", [], []

    def close(falls_to):
        blocks[label] = (lines, ends + ([falls_to] if falls_to else []))
    fresh = 0
    for line in body:
        m = re.match(r"(\.L\w+):", line)
        if m:
            close(m.group(1))
            label, lines, ends = m.group(1), [], []
            continue
        lines.append(line)
        m = BRANCH.match(line)
        if m or "s_endpgm" in line:
            fresh += 1
            if m:
                ends.append(m.group(2))
            go_on = None if "s_endpgm" in line or m.group(1) == "s_branch" else f"after{fresh}"
            close(go_on)
            label, lines, ends = go_on or f"dead{fresh}", [], []
    close(None)
    return blocks


def late_barriers(body):
    """The (block, line) of barriers that a wave may reach with a load to LDS under way, and from which a
    matrix product can be reached (the kernel's loops, not its end)."""
    blocks = blocks_of(body)
    feeds = {b for b, (lines, _) in blocks.items() if any("v_mfma" in x for x in lines)}
    while True:
        more = {b for b, (_, ends) in blocks.items() if any(e in feeds for e in ends)} | feeds
        if more == feeds:
            break
        feeds = more

    def through(lines, pending, at=None):
        for i, x in enumerate(lines):
            if LOAD.match(x):
                pending = True
            elif re.match(r"\s+s_waitcnt\b.*vmcnt\(0\)", x):
                pending = False
            elif at is not None and re.match(r"\s+s_barrier\b", x) and pending:
                at.append(i)
        return pending
    entry = dict.fromkeys(blocks, False)
    while True:
        left = {b: through(lines, entry[b]) for b, (lines, _) in blocks.items()}
        now = dict.fromkeys(blocks, False)
        for b, (_, ends) in blocks.items():
            for e in ends:
                now[e] |= left[b]
        if now == entry:
            break
        entry = now
    late = []
    for b, (lines, ends) in blocks.items():
        at = []
        through(lines, entry[b], at)
        for i in at:
            if any("v_mfma" in x for x in lines[i:]) or any(e in feeds for e in ends):
                late.append((b, i))
    return late


def test_the_search_itself():
    load, wait, barrier = "\tglobal_load_lds_dword v[2:3], off", "\ts_waitcnt vmcnt(0)", "\ts_barrier"
    mfma, end = "\tv_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], 0", "\ts_endpgm"
    assert not late_barriers([load, wait, barrier, mfma, end])
    assert late_barriers([load, barrier, mfma, end]) == [("entry", 1)]
    assert not late_barriers([mfma, load, barrier, end])                # nothing behind it but the end
    loop = [".LBB0_1:", "\ts_cbranch_execz .LBB0_2", wait, ".LBB0_2:", barrier, load, mfma,
            "\ts_cbranch_scc0 .LBB0_1", end]
    assert late_barriers(loop) == [(".LBB0_2", 0)]                      # a wave that skips the wait
    loop[1], loop[2] = loop[2], loop[1]
    assert not late_barriers(loop)


@pytest.fixture(scope="module")
def prompt_kernels():
    src = "pages_prompt.hip"
    r = subprocess.run([B._hipcc(), *B.FLAGS, *B.EXTRA.get(src, []), "--cuda-device-only", "-S",
                        os.path.join(B.CSRC, src), "-o", "-"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found = re.findall(r"^_ZN3ckv\d+pages_prompt_kernelILi(\d+)ELb([01])ELi(\d)E\S*:(.*?)^\.Lfunc_end",
                       r.stdout, re.S | re.M)
    return {(int(d), f == "1", int(w)): body.splitlines()[1:] for d, f, w, body in found}


@pytest.mark.parametrize("waves", [4, 8])
@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
def test_chunks_over_pages_wait_for_what_they_load_to_lds(prompt_kernels, d, fp8, waves):
    body = prompt_kernels[d, fp8, waves]
    assert any(LOAD.match(x) for x in body)
    assert late_barriers(body) == []
