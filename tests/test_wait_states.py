"""Wait states in the built code: between a matrix product and the first
instruction that touches its result, on every path through the code.

A product's result registers are written some issue slots after the product
and nothing in the hardware holds a reader back, so the compiler counts the
slots between the two and fills the gap.  ROCm 7.2 counts them along one path
only where several meet, so the sources settle such products themselves
(`mma_settle`) or order them so that they need not.  This reads the library's own
gfx950 code and takes the shortest path.  The counts are those the compiler itself
leaves in straight code."""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2608_06628_amd import binding as hb

STATES = {"v_mfma_f32_32x32x16_bf16": 12, "v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_32x32x2_f32": 18,
          "v_mfma_f32_16x16x4_f32": 10}
OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if p and os.path.exists(p)), None)
REG = re.compile(r"\b([va])(?:(\d+)\b|\[(\d+):(\d+)\])")
BRANCH = re.compile(r"<[^>]*\+0x([0-9a-f]+)>|<([^>+]*)>")


def code_objects(path):
    """The gfx950 code objects in the library's offload bundles."""
    data = open(path, "rb").read()
    at = 0
    while (at := data.find(b"__CLANG_OFFLOAD_BUNDLE__", at)) >= 0:
        entry = at + 32
        for _ in range(struct.unpack_from("<Q", data, at + 24)[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            name = data[entry + 24:entry + 24 + length]
            entry += 24 + length
            if b"gfx950" in name and size:
                yield data[at + offset:at + offset + size]
        at += 24


def kernels(listing):
    """name -> instructions (text, address), from a disassembly."""
    out, cur = {}, None
    for line in listing.splitlines():
        if line.endswith(">:"):
            cur = out.setdefault(line[line.index("<") + 1:-2], [])
        elif cur is not None and line.startswith("\t"):
            text, _, rest = line.partition("//")
            if rest:  # (else zeros between two functions)
                cur.append((text.strip(), int(rest.split(":")[0], 16), rest))
    return out


def registers(text):
    s = set()
    for kind, one, lo, hi in REG.findall(text):
        s.update((kind, i) for i in (range(int(lo), int(hi) + 1) if lo else (int(one),)))
    return s


def shortest(code):
    """(states, needed, product, reader) of every product whose result is
    touched before it is there."""
    ops = [t.split(None, 1)[0] for t, _, _ in code]
    place = {a: i for i, (_, a, _) in enumerate(code)}
    first = code[0][1]
    regs = {}

    def touched(i):
        if i not in regs:
            text = code[i][0]
            # (the instruction's own accumulator may follow at once: a product adds on to a product)
            ops_ = text.split(None, 1)[1].split(", ") if " " in text else []
            if ops[i].startswith("v_mfma"):
                regs[i] = (registers(", ".join(ops_[1:3])), registers(ops_[0]))
            else:
                regs[i] = (registers(text), set())
        return regs[i]

    def target(i):
        m = BRANCH.search(code[i][2])
        return place[first + int(m.group(1), 16) if m.group(1) else first]

    bad = []
    for i, op in enumerate(ops):
        if not op.startswith("v_mfma"):
            assert "mfma" not in op and "smfmac" not in op, op
            continue
        need, result = STATES[op], touched(i)[1]
        seen, todo = {}, [(i + 1, 0)]
        while todo:
            p, s = todo.pop()
            if p >= len(code) or s >= need or seen.get(p, 99) <= s:
                continue
            seen[p] = s
            if not ops[p].startswith("s_"):
                reads, writes = touched(p)
                if reads & result:
                    bad.append((s, need, code[i][0], code[p][0]))
                    continue
                if writes & result:
                    continue  # adds on: from here that product's own count
            if ops[p] == "s_endpgm":
                continue
            if ops[p] == "s_branch":
                todo.append((target(p), s + 1))
                continue
            if ops[p].startswith("s_cbranch"):
                todo.append((target(p), s + 1))
            todo.append((p + 1, s + (int(code[p][0].split()[1], 0) + 1 if ops[p] == "s_nop" else 1)))
    return bad


def test_results_are_read_when_they_are_there(tmp_path):
    if OBJDUMP is None:
        pytest.skip("no llvm-objdump")
    assert os.path.exists(hb.LIB_PATH), "the library is not built"
    early, products = {}, 0
    for n, obj in enumerate(code_objects(hb.LIB_PATH)):
        f = tmp_path / f"{n}.elf"
        f.write_bytes(obj)
        listing = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(f)], capture_output=True, text=True, check=True).stdout
        for name, code in kernels(listing).items():
            products += sum(t.startswith("v_mfma") for t, _, _ in code)
            if bad := shortest(code):
                early[name] = (len(bad), min(bad))
    assert products > 1000, "no products found: the listing was not understood"
    assert not early, "\n".join(f"{k}: {n} of its products, {b[0]} of {b[1]} states: {b[2]} -> {b[3]}"
                                for k, (n, b) in sorted(early.items()))


def test_the_shortest_way_counts():
    """A product's reader behind a block that is passed by."""
    text = """
0000000000000000 <kernel>:
\tv_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]// 000000000000: 00000000 00000000
\ts_cbranch_scc0 1                                           // 000000000008: 00000000 <kernel+0x10>
\ts_nop 7                                                    // 00000000000C: 00000000
\tv_mfma_f32_16x16x32_bf16 a[16:19], v[0:3], v[4:7], 0       // 000000000010: 00000000 00000000
\ts_nop %d                                                    // 000000000018: 00000000
\tv_accvgpr_read_b32 v8, a15                                 // 00000000001C: 00000000 00000000
\ts_endpgm                                                   // 000000000024: 00000000
"""
    code = kernels(text % 1)["kernel"]
    assert [b[:2] for b in shortest(code)] == [(4, 12)]
    assert shortest(kernels(text % 9)["kernel"]) == []
    feeds = text.replace("v[0:3], v[4:7], 0 ", "a[0:3], v[4:7], 0 ")  # the product as another's operand
    assert min(shortest(kernels(feeds % 9)["kernel"]))[:2] == (1, 12)
