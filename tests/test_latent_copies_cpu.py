"""Copies into LDS of the absorbed latent attention, read from the machine code that the library was built to: on no path
does a wave write results, or end, with a copy under way.  A tile's results leave behind the barrier that gives its buffers
to the next tile, so a copy that is still under way there could land on the next tile's queries (or after the CTA's end)."""
from __future__ import annotations

import os
import re
import subprocess

import pytest

from paper_2606_13392_amd import build, msa

LLVM = os.path.join(os.path.dirname(os.path.dirname(build.HIPCC)), "llvm", "bin")


def _code_objects(path):
    """The gfx950 code objects of a shared library: bundles, one per source file."""
    data = open(path, "rb").read()
    at = data.find(b"__CLANG_OFFLOAD_BUNDLE__")
    while at >= 0:
        p = at + 32
        for _ in range(int.from_bytes(data[at + 24:p], "little")):
            offset, size, name = (int.from_bytes(data[p + 8 * i:p + 8 * i + 8], "little") for i in range(3))
            if b"gfx950" in data[p + 24:p + 24 + name] and size:
                yield data[at + offset:at + offset + size]
            p += 24 + name
        at = data.find(b"__CLANG_OFFLOAD_BUNDLE__", p)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: [(address, instruction)]} of the absorbed attention's kernels."""
    msa.lib()
    found = {}
    for i, obj in enumerate(_code_objects(build.LIB)):
        if b"latent_paged_kernel" not in obj:
            continue
        f = tmp_path_factory.mktemp("code") / f"{i}.co"
        f.write_bytes(obj)
        text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", str(f)], check=True,
                              capture_output=True, text=True).stdout
        name = None
        for line in text.splitlines():
            head = re.match(r"^[0-9a-f]+ <(.+)>:", line)
            code = re.match(r"^\s+(\S.*?)\s*//\s*([0-9A-F]+):", line)
            if head:
                name = head.group(1)
            elif code and name and "latent_paged_kernel" in name:
                found.setdefault(name, []).append((int(code.group(2), 16), code.group(1)))
    return found


def under_way(code):
    """For each instruction, whether some path reaches it with a copy into LDS that was not waited for."""
    index = {a: i for i, (a, _) in enumerate(code)}
    state = [None] * len(code)
    state[0], todo = False, [0]
    while todo:
        i = todo.pop()
        address, text = code[i]
        op = text.split()[0]
        assert op not in ("s_setpc_b64", "s_swappc_b64"), "a call: paths cannot be followed"
        copies = state[i]
        if op.startswith("global_load_lds"):
            copies = True
        elif op == "s_waitcnt" and "vmcnt(0)" in text:
            copies = False
        then = [] if op in ("s_endpgm", "s_branch") else [i + 1]
        if op == "s_branch" or op.startswith("s_cbranch"):
            off = int(text.split()[1])
            then.append(index[address + 4 + 4 * (off - (1 << 16) if off >= 1 << 15 else off)])
        for j in then:
            if state[j] is None or (copies and not state[j]):
                state[j] = copies
                todo.append(j)
    return state


def test_no_copy_is_under_way_where_results_leave(kernels):
    assert len(kernels) == 4                                # two cache types, two latent sizes
    for name, code in kernels.items():
        state = under_way(code)
        ends = [(s, t) for s, (_, t) in zip(state, code) if t.startswith(("global_store", "s_endpgm"))]
        assert any(t.startswith("global_load_lds") for _, t in code) and len(ends) > 2
        late = [t for s, t in ends if s]
        assert not late, f"{name}: {len(late)} of {len(ends)}, e.g. {late[0]}"
