"""What the assembly of the gated products has to keep, because loads straight into LDS are written in assembly and nobody else counts them or
sees to their operands: faults here would show on the GPU only now and then."""
import re
import subprocess

import pytest

from paper_2507_07149_amd import build

LDS_LOAD = re.compile(r"buffer_load_dwordx4 v\d+, s\[(\d+):(\d+)\], 0 offen lds")
OTHER_MEMORY = re.compile(r"(global|flat|scratch|buffer)_(load|store|atomic)")


@pytest.fixture(scope="module")
def functions():
    """{kernel: its instructions, without comments; labels end in a colon}"""
    defines = next(s for s in build.SOURCES if s[1] == "gated_product_bf16")[2]
    r = subprocess.run([build.HIPCC, *build.FLAGS, *defines, "--cuda-device-only", "-S", build.CSRC + "/gated_product.hip", "-o", "-"],
                       stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    out, cur = {}, None
    for line in r.stdout.splitlines():
        s = line.split(";")[0].strip()
        if m := re.match(r"(_Z\w*k_gated_\w+):", s):
            cur = out.setdefault(m.group(1), [])
        elif s.startswith(".Lfunc_end"):
            cur = None
        elif cur is not None and s and (not s.startswith(".") or s.endswith(":")):
            cur.append(s)
    return out


def test_buffers_of_loads_come_from_the_scalar_unit(functions):
    """A buffer's registers written by the vector unit are seen by a memory instruction five cycles later; the compiler waits for instructions that
    it knows, not for those in assembly blocks."""
    loads = 0
    for name, code in functions.items():
        for i, s in enumerate(code):
            m = LDS_LOAD.match(s)
            if not m:
                continue
            loads += 1
            buffer, waited = set(range(int(m.group(1)), int(m.group(2)) + 1)), 0
            for before in reversed(code[max(i - 12, 0):i]):
                if waited >= 5:
                    break
                written = re.match(r"v_\S+ s\[?(\d+)(?::(\d+))?\]?,", before)
                if written:
                    assert not buffer & set(range(int(written.group(1)), int(written.group(2) or written.group(1)) + 1)), (name, before, s)
                nop = re.match(r"s_nop (\d+)", before)
                waited += int(nop.group(1)) + 1 if nop else 0 if before.endswith(":") else 1
    assert loads > 500


def _loops(code):
    """The instructions of each loop with matrix instructions: blocks that lead to each other."""
    starts = sorted({0} | {i for i, c in enumerate(code) if c.endswith(":")} | {i + 1 for i, c in enumerate(code) if c.startswith(("s_cbranch", "s_branch"))})
    blocks = [code[a:b] for a, b in zip(starts, starts[1:] + [len(code)])]
    labels = {b[0][:-1]: n for n, b in enumerate(blocks) if b and b[0].endswith(":")}
    after = []
    for n, b in enumerate(blocks):
        last = b[-1] if b else ""
        to = [labels[last.split()[-1]]] if last.startswith(("s_cbranch", "s_branch")) else []
        after.append(to + ([n + 1] if not last.startswith(("s_branch", "s_endpgm")) and n + 1 < len(blocks) else []))

    def reached(n):
        seen, rest = set(), list(after[n])
        while rest:
            if (b := rest.pop()) not in seen:
                seen.add(b)
                rest += after[b]
        return seen

    reach = [reached(n) for n in range(len(blocks))]
    loops = {frozenset(b for b in reach[n] if n in reach[b]) for n in range(len(blocks)) if n in reach[n]}
    bodies = [[s for b in sorted(loop) for s in blocks[b]] for loop in loops]
    return [body for body in bodies if any("v_mfma" in s for s in body)]


def test_loops_of_products_wait_for_their_own_loads(functions):
    """A wait in front of a barrier leaves the loads of the steps ahead in flight: all buffers but the one that is read and the one that is filled next.
    It counts them right if a step issues as many as it should, and if the loop has no other access to memory."""
    products = {n: c for n, c in functions.items() if re.search("k_gated_(product|gradients)", n)}
    assert len(products) == 4 * 4 + 4                          # kinds in four tiles each, gradients side by side in each
    for name, code in products.items():
        tile = re.search(r"TileILi(\d+)ELi(\d+)ELi2ELi2ELi(\d+)E", name)
        if tile:                                               # four waves, a kilobyte to a load
            rows, cols, buffers = map(int, tile.groups())
            step = (rows + cols) // 8 // 4
            ahead = (buffers - 2) * step
        else:                                                  # 256 x 256, half a step ahead
            step, ahead = 16, 8
        loops = _loops(code)
        assert len(loops) >= (2 if "gradients" in name else 1), name
        for loop in loops:
            assert not [s for s in loop if OTHER_MEMORY.match(s) and not LDS_LOAD.match(s)], name
            barriers = sum(1 for s in loop if s.startswith("s_barrier"))
            waits = [int(m.group(1)) for s in loop if (m := re.search(r"s_waitcnt.*vmcnt\((\d+)\)", s))]
            assert sum(1 for s in loop if LDS_LOAD.match(s)) == step * barriers > 0, name
            assert waits.count(ahead) == barriers and set(waits) <= {0, ahead}, (name, waits)


def test_sums_are_left_alone_next_to_their_products(functions):
    """Products are written in assembly too, so the compiler does not keep others away from their sums: a sum is read or written by another instruction
    only 11 wait states or more behind a product that writes it, and by a product two or more behind another that writes it."""
    registers = lambda s: {r for m in re.finditer(r"\ba(?:\[(\d+):(\d+)\]|(\d+))", s)
                           for r in range(int(m.group(1) or m.group(3)), int(m.group(2) or m.group(3)) + 1)}
    products = 0
    for name, code in functions.items():
        now, product, other = 0, {}, {}
        for s in code:
            if s.endswith(":"):
                continue
            sums = registers(s)
            if s.startswith("v_mfma"):
                products += 1
                assert all(now - other.get(r, -99) > 2 for r in sums), (name, s)
                product.update((r, now) for r in sums)
            elif sums:
                assert all(now - product.get(r, -99) > 11 for r in sums), (name, s)
                if re.match(r"v_accvgpr_(write|mov)", s):
                    other.update((r, now) for r in registers(s.split(",")[0]))
            nop = re.match(r"s_nop (\d+)", s)
            now += int(nop.group(1)) + 1 if nop else 1
    assert products > 1000
