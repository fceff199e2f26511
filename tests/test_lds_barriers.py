"""Waits in front of barriers, from the built kernels' own instructions (no GPU).

What wavefronts exchange through LDS is there behind a barrier only if each of them waited for its LDS operations in front of it (s_waitcnt lgkmcnt(0)).  The
compiler derives that wait from the fence at the barrier, and drops it where a loop begins with the barrier and nothing is outstanding when the loop is entered, also
if the way back to its beginning leaves writes outstanding.
"""
import re
import shutil
import subprocess

import pytest

from paper_2010_15884_amd import binding as B
from paper_2010_15884_amd import build

LLVM = "/opt/rocm/llvm/bin"

# Kernels whose barriers may find LDS operations outstanding, and why that is harmless.
HARMLESS = {
    # on the way from one columns' sums to the next: writes of a lane to places that it alone writes next, and that others read behind a further barrier
    "norm_grad_sums_kernel": 1,
}


def outstanding(instructions, target):
    """The barriers that may be reached with LDS operations under way: {place: operations}.  instructions: [(place, text)] of a kernel in order; target(i): the index that
    the branch at index i goes to.  Of the LDS operations (which end in their order, beside scalar loads) a wait for n leaves at most n."""
    leaders = {0} | {i + 1 for i, (_, t) in enumerate(instructions) if t.startswith(("s_cbranch", "s_branch", "s_endpgm"))}
    leaders |= {target(i) for i, (_, t) in enumerate(instructions) if t.startswith(("s_cbranch", "s_branch"))}
    leaders = sorted(i for i in leaders if i < len(instructions))
    ends = dict(zip(leaders, leaders[1:] + [len(instructions)]))

    def run(begin, pending, found=None):
        """Through a block: the most LDS operations that are outstanding behind it."""
        for i in range(begin, ends[begin]):
            place, text = instructions[i]
            if text.startswith("ds_"):
                pending += 1
            elif text.startswith("s_waitcnt"):
                wait = re.search(r"lgkmcnt\((\d+)\)", text)
                if wait:
                    pending = min(pending, int(wait[1]))
            elif text.startswith("s_barrier") and pending and found is not None:
                found[place] = pending
        return min(pending, 16)
    entry, work, found = {0: 0}, [0], {}
    while work:
        begin = work.pop()
        behind = run(begin, entry[begin])
        i = ends[begin] - 1
        text = instructions[i][1]
        after = [target(i)] if text.startswith(("s_cbranch", "s_branch")) else []
        if not text.startswith(("s_branch", "s_endpgm")) and i + 1 < len(instructions):
            after.append(i + 1)
        for b in after:
            if b not in entry or behind > entry[b]:
                entry[b] = behind
                work.append(b)
    for begin, pending in entry.items():
        run(begin, pending, found)
    return found


def _disassembled(tmp):
    """{kernel: {place: operations}} of the built library's kernels that have a barrier."""
    fat, obj = str(tmp / "fat"), str(tmp / "code.o")
    subprocess.run([f"{LLVM}/llvm-objcopy", f"--dump-section=.hip_fatbin={fat}", B.LIB_PATH, str(tmp / "unused")], check=True)
    data = open(fat, "rb").read()
    starts = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)]
    kernels = {}
    for a, b in zip(starts, starts[1:] + [len(data)]):
        open(fat, "wb").write(data[a:b])
        subprocess.run([f"{LLVM}/clang-offload-bundler", "--type=o", "--unbundle", f"--input={fat}", f"--output={obj}",
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True)
        text = subprocess.run([f"{LLVM}/llvm-objdump", "-d", obj], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"^(?=[0-9a-f]+ <)", text, flags=re.M):
            head = re.match(r"([0-9a-f]+) <(\w+)>:", part)
            if not head or "s_barrier" not in part:
                continue
            lines = re.findall(r"^\s+(\S.*?)\s*// ([0-9A-F]+):[^<\n]*(?:<\w+(?:\+0x([0-9a-f]+))?>)?$", part, re.M)
            base = int(head[1], 16)
            instructions = [(int(at, 16) - base, t) for t, at, _ in lines]
            index = {place: i for i, (place, _) in enumerate(instructions)}
            goes = {i: index[int(to or "0", 16)] for i, (t, _, to) in enumerate(lines) if t.startswith(("s_cbranch", "s_branch"))}
            kernels[head[2]] = outstanding(instructions, goes.__getitem__)
    return kernels


def test_the_reading_itself():
    """A loop that begins with a barrier and ends with a write, without and with a wait; a wait that leaves one operation; two ways to one barrier."""
    loop = [(0, "s_barrier"), (4, "ds_read_b32 v0, v1"), (8, "s_waitcnt lgkmcnt(0)"), (12, "s_barrier"), (16, "ds_write_b32 v1, v0"), (20, "s_cbranch_scc1 0"), (24, "s_endpgm")]
    assert outstanding(loop, {5: 0}.__getitem__) == {0: 1}
    assert outstanding([(-4, "s_waitcnt vmcnt(0) lgkmcnt(0)"), *loop], {6: 0}.__getitem__) == {}
    line = [(0, "ds_read_b32 v0, v1"), (4, "ds_read_b32 v2, v1"), (8, "s_waitcnt lgkmcnt(1)"), (12, "s_barrier"), (16, "s_waitcnt lgkmcnt(0)"), (20, "s_barrier"), (24, "s_endpgm")]
    assert outstanding(line, None) == {12: 1}
    ways = [(0, "s_cbranch_scc0 2"), (4, "ds_write_b32 v1, v0"), (8, "s_barrier"), (12, "s_endpgm")]
    assert outstanding(ways, {0: 2}.__getitem__) == {8: 1}


def test_built_kernels_wait_in_front_of_their_barriers(tmp_path):
    kernels = _disassembled(tmp_path)
    assert len(kernels) > 100 and sum("delta_" in n for n in kernels) > 30
    late = {n: f for n, f in kernels.items() if f and not any(name in n and len(f) <= most for name, most in HARMLESS.items())}
    assert not late, late


@pytest.mark.parametrize("header", ["delta_tile.h", "matrix_blocks.h"])
def test_a_loop_that_begins_with_the_barrier(tmp_path, header):
    """The form in which the compiler drops the fence's wait."""
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc is not installed")
    source = tmp_path / "loop.hip"
    source.write_text(f"""#include <hip/hip_runtime.h>
#include "{header}"
__global__ void loop(float* x, int n)
{{
    __shared__ float a[256];
    float v = x[threadIdx.x];
    if (n > 0) {{
        a[threadIdx.x] = v;
        sysconv::lds_barrier();
    }}
    for (int i = n; i > 0; --i) {{
        sysconv::lds_barrier();
        v += a[(threadIdx.x + 77) & 255];
        sysconv::lds_barrier();
        a[threadIdx.x] = v;
    }}
    x[threadIdx.x] = v;
}}
""")
    got = subprocess.run(["hipcc", *[f for f in build.FLAGS if f not in ("-Wall", "-Wextra")], "--cuda-device-only", "-S", str(source), "-o", "-"], capture_output=True,
                         text=True, check=True).stdout
    body = re.search(r"^_Z4loop\w+:(.*?)^\.Lfunc_end", got, re.M | re.S)[1]
    instructions, labels, names = [], {}, {}
    for line in body.splitlines():
        line = line.split(";")[0].strip()
        if line.endswith(":"):
            labels[line[:-1]] = len(instructions)
        elif line and not line.startswith("."):
            if line.startswith(("s_cbranch", "s_branch")):
                names[len(instructions)] = line.split()[1]
            instructions.append((len(instructions), line))
    assert sum(t.startswith("s_barrier") for _, t in instructions) == 3
    assert outstanding(instructions, lambda i: labels[names[i]]) == {}
