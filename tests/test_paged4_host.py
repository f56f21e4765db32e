"""Host side of the 4-bit pages and of appends with rotary positions (CPU): argument blocks are laid out as
fkv.h has them, refusals come back from the C entry before anything is launched, and the kernels' waits are voted on."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_07144_gb300", "csrc")


def test_the_argument_block_is_laid_out_as_the_struct(tmp_path):
    from paper_2607_07144_gb300 import _binding
    fields = ["q", "q_out", "k", "v", "slots", "pos", "cos", "sin", "q_stride_tok", "q_stride_head", "out_stride_tok",
              "out_stride_head", "k_stride_tok", "k_stride_head", "v_stride_tok", "v_stride_head", "table_stride", "n_pos",
              "n_tok", "dtype", "n_q_heads", "rot", "interleaved"]
    src = tmp_path / "a.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "fkv.h"\nint main(void) {\n' +
                   "".join('printf("%%zu ", offsetof(fkv_rotary, %s));\n' % f for f in fields) +
                   'printf("%zu %d %d %d\\n", sizeof(fkv_rotary), FKV_E4M3, FKV_INT8, FKV_UINT4);\nreturn 0; }\n')
    exe = tmp_path / "a"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    sizes = {"P": 8, "q": 8, "i": 4}
    at, want = 0, []
    for n, c in re.findall(r"(\d+)([Pqi])", _binding._ROTARY.format):
        for _ in range(int(n)):
            want.append(at)
            at += sizes[c]
    assert got[:len(fields)] == want and got[len(fields)] == at == _binding._ROTARY.size
    assert got[-3:] == [_binding.E4M3, _binding.INT8, _binding.UINT4]


def test_calls_without_a_context_are_refused():
    from paper_2607_07144_gb300 import _binding, build
    build.build()
    L = _binding.lib()
    buf = ctypes.create_string_buffer(_binding._ROTARY.size)
    assert L.fkv_page_append(None, None, buf, None) == _binding.EINVAL


def test_waits_are_voted_on():
    """As in k_attend_step: a lane that gives up takes its warp along, and loads in flight get a while to land."""
    t = open(os.path.join(CSRC, "attend4.cu")).read()
    waits = [m.start() for m in re.finditer(r"mbar_wait\(", t)]
    assert len(waits) == 2 and sum(t[:w].endswith("__all_sync(~0u, ") for w in waits) == 1
    assert "a.status, 2000000);\n            __syncwarp();" in t


def test_every_warp_of_a_group_gives_up_registers_by_one_instruction():
    """setmaxnreg is for all warps of a group at once: no role that only some of them have holds one."""
    t = open(os.path.join(CSRC, "attend_prompt.cu")).read()
    found = re.findall(r"([^\n]*)\n\s*asm volatile\(\"setmaxnreg", t)
    assert [x.strip() for x in found] == ["if (FOUR && group >= 2)", "if (!FOUR)", "if constexpr (!FOUR) {", "} else {"]


@pytest.mark.parametrize("rows,want", [(8, 3), (16, 2)])
def test_blocks_and_shared_memory_fit(rows, want):
    """The shared memory of as many blocks as the plan counts on an SM is there (228 KB, 1 KB of each the system's)."""
    t = open(os.path.join(CSRC, "attend.cuh")).read()
    assert "constexpr int kStep4Keys = 64;" in t and "step4_blocks(int nt) { return nt == 1 ? 3 : 2; }" in t
    nt, most = rows // 8, 0
    for D, stages in ((128, 2), (64, 3)):
        ring = 4 * stages * (2 * 4 * 8 * D + 2 * 4 * 64)
        smem = ring + (nt * (D // 16) * 256 if nt > 1 else 0) + 4 * 64 * 20 + 4 * 2 * rows * 4 + 1024
        most = max(most, smem + 256 + 1024)                # static arrays, the system's
    assert want * most <= 228 * 1024
