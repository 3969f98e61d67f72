"""What libwsattn.so exports beside its C ABI: nothing of the host side's checks
and plans, which a program's own function of the same name would replace."""
import subprocess

import paper_2606_25041_amd as ws
from paper_2606_25041_amd import build

# the host side's calls into the kernels' sources (csrc/ws_kernels.h)
LAUNCHERS = {"launch_attention", "launch_combine", "launch_append", "launch_append4", "launch_read4", "launch_few4",
             "launch_prefill_bwd", "current_device_cus", "scratch_address"}


def test_only_the_abi_and_the_launchers():
    ws.library()
    out = subprocess.run(["nm", "-D", "--defined-only", "--demangle", build.LIB], capture_output=True, text=True, check=True).stdout
    names = [ln.split(" ", 2)[2] for ln in out.splitlines()]
    inner = {n.split("(")[0].split("::")[-1] for n in names if "ws::" in n}
    assert any(n.startswith("ws_block_causal_attn_fwd") for n in names)
    assert inner <= LAUNCHERS, sorted(inner - LAUNCHERS)
