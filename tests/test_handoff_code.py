"""Kernels whose last workgroup to finish goes on with what the others wrote: between a wave's stores and its
workgroup's arrival at the counter the wave has to wait for them itself.  A barrier waits for LDS only, and the fence
and the count of one thread order its own wave's memory; a store of another wave that is still on its way could land
after the last workgroup, on another die, has read the word.  No run shows this reliably, so the check is on the gfx950
code that the library's own flags produce, without a GPU."""
import os
import re
import subprocess

import pytest

import paper_2602_06502_amd._build as B

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def _kernels(tmp_path, source):
    """Kernel name -> its instructions."""
    if not os.path.exists(B.HIPCC) or not os.path.exists(OBJDUMP):
        pytest.skip("ROCm compiler tools not installed")
    obj = str(tmp_path / "code.o")
    r = subprocess.run([B.HIPCC, *B.FLAGS, "--cuda-device-only", "--no-gpu-bundle-output", "-c",
                        os.path.join(B.CSRC, source), "-o", obj], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    out = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", obj], stdout=subprocess.PIPE, text=True, check=True).stdout
    kernels, name = {}, None
    for line in out.splitlines():
        m = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        if m:
            name = m.group(1)
            kernels[name] = []
        elif name and line.startswith("\t"):
            kernels[name].append(line.split("//")[0].strip())
    return kernels


MEMORY = re.compile(r"(global|flat|buffer|scratch)_(?!inv|wbl2)")


@pytest.mark.timeout(600)
@pytest.mark.parametrize("source,kernel", [("dm_attn.hip", "attn_plan_kernel"), ("dm_pages.hip", "fork_scan_kernel")])
def test_waves_wait_for_their_stores_before_they_arrive(tmp_path, source, kernel):
    code = [v for k, v in _kernels(tmp_path, source).items() if kernel in k]
    assert len(code) == 1
    code = code[0]
    releases = [i for i, x in enumerate(code) if x.startswith("buffer_wbl2 sc1")]
    # the release by one thread, then its count
    hands = [i for i in releases if any(x.startswith("global_atomic_add") and "sc0" in x for x in code[i:i + 20])]
    assert len(hands) == 1, hands
    barrier = max(i for i in range(hands[0]) if code[i].startswith("s_barrier"))
    for i in range(barrier - 1, -1, -1):
        m = re.match(r"s_waitcnt .*vmcnt\((\d+)\)", code[i])
        if m and int(m.group(1)) == 0:
            return
        assert not MEMORY.match(code[i]), ("an access after the last wait before the barrier", code[i])
        assert not re.match(r"s_(c?branch|setpc|swappc|barrier)", code[i]), ("no wait before the barrier", code[i:barrier + 1])
    raise AssertionError("no wait before the barrier")
