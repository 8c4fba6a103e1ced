"""What the compiler cannot see to in assembly strings, looked for in the library as it was built:
wait states that the hardware does not insert.

Two of CDNA's rules concern the direct loads to LDS, which the kernels write as assembly strings
(m0 holds the LDS address, the base may be scalar):
  - a scalar write of m0, then an LDS load that reads it: one wait state between them
  - a vector instruction's write of a scalar register (readfirstlane, readlane, a comparison), then
    a memory instruction that reads it: five
Every instruction in between counts as one, s_nop n as n + 1."""
import collections
import os
import re
import shutil
import struct
import subprocess

import pytest

import paper_2606_01556_amd as tq

OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if p and os.path.exists(p)), None)
LIB = os.path.join(os.path.dirname(tq.__file__), "libtq.so")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def scalars(text):
    """The scalar registers that an operand list names."""
    out = {int(m) for m in re.findall(r"\bs(\d+)\b", text)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        out.update(range(int(a), int(b) + 1))
    return out


def written_by_vector(op, args):
    """Scalar registers that a vector instruction writes: its first operand, the carry its second."""
    parts = re.split(r",\s*(?![^\[]*\])", args)
    out = scalars(parts[0]) if parts[0].startswith("s") else set()
    if op.startswith(("v_add_co", "v_sub_co", "v_subrev_co", "v_addc_co", "v_subb_co", "v_div_scale", "v_mad_u64", "v_mad_i64")):
        out |= scalars(parts[1])
    return out


def hazards(lines):
    """(kind, kernel, instruction) of every memory instruction that comes too early behind a write
    of what it reads, in the order of the code."""
    kernel, before = "", collections.deque(maxlen=8)
    for line in lines:
        label = re.search(r"<(\S+)>:", line)
        if label:
            if not label[1].startswith("L"):
                kernel = label[1]
                before.clear()
            continue
        op, _, args = line.split("//")[0].strip().partition(" ")
        if not op or op.startswith((".", "/")):
            continue
        args = args.strip()
        if op.startswith(("global_", "buffer_", "flat_", "scratch_")):
            reads, states = scalars(args), 0
            for o, a in reversed(before):
                first = a.split(",")[0].strip()
                if "_lds_" in op and o.startswith("s_") and first == "m0" and states < 1:
                    yield "m0", kernel, f"{o} {a}; {op} {args}"
                if o.startswith("v_") and written_by_vector(o, a) & reads:
                    yield "scalar", kernel, f"{o} {a}; {op} {args}"
                elif o.startswith("s_"):
                    reads -= scalars(first)          # (the newer write is the one that is read)
                states += int(a, 0) + 1 if o == "s_nop" else 1
                if states >= 5:
                    break
        before.append((op, args))


def code_objects():
    """The code objects of the library: offload bundles behind each other."""
    data, at = open(LIB, "rb").read(), 0
    while (at := data.find(MAGIC, at)) >= 0:
        count, place = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, place)
            name = data[place + 24:place + 24 + length].decode()
            place += 24 + length
            if size and name.endswith("gfx950"):
                yield data[at + offset:at + offset + size]
        at += len(MAGIC)


@pytest.mark.parametrize("code, found", [
    ("s_mov_b32 m0, s1\nglobal_load_lds_dwordx4 v0, s[2:3]", ["m0"]),
    ("s_mov_b32 m0, s1\ns_nop 0\nglobal_load_lds_dwordx4 v0, s[2:3]", []),
    ("s_mov_b32 m0, s1\nv_mov_b32_e32 v9, v8\nglobal_load_lds_dwordx4 v0, off", []),
    ("v_readfirstlane_b32 s3, v1\ns_mov_b32 m0, s1\ns_nop 0\nglobal_load_lds_dwordx4 v0, s[2:3]", ["scalar"]),
    ("v_readfirstlane_b32 s3, v1\ns_mov_b32 m0, s1\ns_nop 3\nglobal_load_lds_dwordx4 v0, s[2:3]", []),
    ("v_readlane_b32 s2, v1, 7\ns_add_u32 s2, s4, s5\ns_nop 0\nglobal_load_dword v0, v1, s[2:3]", []),
    ("v_cmp_gt_f32_e64 s[2:3], v1, v2\nglobal_load_dword v0, v1, s[2:3]", ["scalar"]),
    ("v_add_co_u32_e64 v4, s[2:3], v1, v2\nglobal_load_dword v0, v1, s[2:3]", ["scalar"]),
])
def test_the_search_itself(code, found):
    assert [kind for kind, _, _ in hazards(("0 <k>:\n" + code).splitlines())] == found


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
@pytest.mark.skipif(not os.path.exists(LIB), reason="libtq.so is not built")
def test_direct_loads_wait(tmp_path):
    objects = list(code_objects())
    assert objects
    loads, bad = 0, []
    for i, obj in enumerate(objects):
        path = tmp_path / f"{i}.co"
        path.write_bytes(obj)
        out = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(path)], check=True,
                             capture_output=True, text=True).stdout
        path.unlink()
        loads += out.count("global_load_lds_dwordx4")
        bad += hazards(out.splitlines())
    assert loads > 0
    assert not bad, f"{len(bad)} loads come too early, the first: {bad[:3]}"
