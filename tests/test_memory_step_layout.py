"""The single step's LDS (csrc/memory_shape.h): B and C are read as 16-byte pieces, so they begin at 16 bytes for every head size and every
number of waves a head (C behind a state of whole pieces), and nothing overlaps."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_09237_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "memory_shape.h"
int main() {
    long n = 0, wrong = 0;
    for (int p = 1; p <= 64; ++p)
        for (int s = 1; s <= 64; ++s)
            for (int parts = 1; parts <= 4; parts += 3) {
                const StepLayout l = step_layout(p, s, parts);
                ++n;
                wrong += l.b % 4 != 0 || l.wave % 4 != 0 || l.each * parts < p || l.b < l.each || l.wave < l.b + 2 * s;
            }
    printf("layouts %ld wrong %ld\n", n, wrong);
    return wrong ? 1 : 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")
def test_parts_begin_at_sixteen_bytes(tmp_path):
    src, exe = tmp_path / "p.cpp", tmp_path / "p"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I" + CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


# a state of whole pieces beside a head (or a quarter of it) that is none, few heads (four waves each) and many
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("N,H,P,G,S,W", [(3, 4, 9, 1, 16, 4), (2, 3, 10, 1, 64, 3), (5, 2, 37, 2, 64, 4), (1, 1, 1, 1, 4, 2), (400, 4, 9, 2, 64, 4),
                                         (520, 3, 37, 1, 16, 4), (800, 2, 10, 1, 20, 2), (1600, 1, 63, 1, 12, 4)])
def test_step(N, H, P, G, S, W, dtype):
    import torch
    from paper_2603_09237_amd import binding
    from test_gpu_memory import _kind, close, conv_definition, parts, scan_definition, scan_problem
    dims, h, d = scan_problem(1, N, H, P, G, S, dtype, 0.2, True, seed=N + P)
    C = H * P + 2 * G * S
    g = torch.Generator().manual_seed(1)
    w, b, cin = torch.randn(C, W, generator=g) * W ** -0.5, torch.randn(C, generator=g), torch.randn(N, W - 1, C, generator=g).to(_kind(dtype))
    conv, seen = conv_definition(h["xbc"].double(), w.double(), b.double(), h["first"], cin.double(), 1)
    x, bb, cc = parts(conv, dims)
    y, last = scan_definition(x.reshape(1, N, H, P), bb.reshape(1, N, G, S), cc.reshape(1, N, G, S), h["dt"].double(), h["z"].double().reshape(1, N, H, P),
                              h["a_log"].double(), h["d"].double(), h["bias"].double(), h["first"], h["state"].double())
    out, state = torch.full((N, W - 1, C), 7.0, dtype=_kind(dtype), device="cuda"), torch.empty_like(d["state"])
    binding.memory_step(dims, W, d["xbc"], d["dt"], d["z"], w.cuda(), b.cuda(), d["a_log"], d["d"], d["bias"], d["first"], cin.cuda(), d["state"], d["y"],
                        out, state)
    close(d["y"], y.reshape(1, N, H * P), S + 16, dtype == 1, "y")
    close(state, last, 16, False, "state")
    assert torch.equal(out.double().cpu(), seen)
