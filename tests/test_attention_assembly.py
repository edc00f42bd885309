"""The loads straight into LDS of attention with a window are written in assembly: the compiler neither sees that they read scalar registers, which must
not come out of the vector unit in the five cycles before, nor counts them in its waits.  The assembly shows both."""
import re
import subprocess

import pytest

from paper_2507_07149_amd import build

SOURCES = ("window_attention", "window_attention_backward", "window_attention_step")


@pytest.fixture(scope="module")
def kernels():
    """{mangled name: instructions, without comments} of every kernel."""
    found = {}
    runs = [subprocess.Popen([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", f"{build.CSRC}/{name}.hip", "-o", "-"], stdout=subprocess.PIPE,
                             stderr=subprocess.DEVNULL, text=True) for name in SOURCES]
    for run in runs:
        text, _ = run.communicate()
        assert run.returncode == 0
        cur = None
        for line in text.splitlines():
            m = re.match(r"(_Z\w*k_(?:window|attention)\w*):", line)
            if m:
                cur = found.setdefault(m.group(1), [])
                continue
            s = line.split(";")[0].strip()
            if line.strip().startswith(".Lfunc_end"):
                cur = None
            elif cur is not None and s and not (s.startswith(".") and not s.startswith(".LBB")):
                cur.append(s)
    return found


def _is_fetch(s):
    return s.startswith("buffer_load") and s.endswith("lds")


def test_buffers_are_old_enough(kernels):
    seen = 0
    for name, code in kernels.items():
        for i, s in enumerate(code):
            if _is_fetch(s):
                assert code[i - 1] == "s_nop 4" and re.match(r"s_mov_b32 m0, (s\d+|vcc_lo|vcc_hi)$", code[i - 2]), (name, code[i - 3:i + 1])
                assert re.search(r", s\[\d+:\d+\], 0 offen lds$", s), (name, s)
                seen += 1
    assert seen > 400


def test_counted_waits_leave_only_the_loads_behind_them(kernels):
    """A wait that lets n loads stay on their way stands right behind n loads of the next tile, in a straight line with them."""
    counted = 0
    for name, code in kernels.items():
        if not any(kind in name for kind in ("k_attention_step", "k_attention_grad_sinks", "_few")):
            assert not any(re.match(r"s_waitcnt vmcnt\([1-9]\d*\)$", s) and _is_fetch(code[i - 1]) for i, s in enumerate(code)), name
            continue
        seen = 0
        for i, s in enumerate(code):
            m = re.match(r"s_waitcnt vmcnt\((\d+)\)( lgkmcnt\(0\))?$", s)
            if not m or int(m.group(1)) == 0:
                continue
            back, loads = i - 1, 0
            while not code[back].startswith((".LBB", "s_cbranch", "s_branch", "s_waitcnt vmcnt(0)")):
                loads += _is_fetch(code[back])
                back -= 1
            if loads == 0:
                continue                                                   # the compiler's own, for its own loads
            assert loads >= int(m.group(1)), (name, loads, s)
            seen += 1
        assert seen >= 1, name
        counted += 1
    assert counted == 4 * 4 * 2                                            # four kernels, four widths, two formats
