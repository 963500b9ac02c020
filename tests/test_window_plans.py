"""How window attention's calls are cut into blocks and wavefronts, asked of the library's own planning code by a small host program."""
import os
import re
import subprocess

import pytest

from paper_2503_06671_amd import binding
from tests.test_abi_host import ROOT, kernel_notes, lib  # noqa: F401

HIPCC = "/opt/rocm/bin/hipcc"
CSRC = os.path.join(ROOT, "paper_2503_06671_amd", "csrc")

PROGRAM = r"""
#include <stdio.h>
#include "esc_window.hip"
// lines of numbers in: N H W heads kv_heads head_dim win_h win_w n_edges f32; a line of name=value words for each pass out
static void show(const char *pass, bool fits, const WindowParams &p, bool f32, int resident)
{
    printf("pass=%s fits=%d tiles=%d ksplit=%d owners=%d waves=%d blocks=%d units=%d chunk=%d tokens=%ld resident=%d\n", pass, fits, p.tiles, p.ksplit,
           p.owners, p.waves, p.blocks, p.units, win_chunk(f32, dim_padded(p.d)), (long)p.wh * in_pairs(p.ww), resident);
}
int main()
{
    esc_window_attn a{};
    int f32;
    while (scanf("%d %d %d %d %d %d %d %d %d %d", &a.N, &a.H, &a.W, &a.heads, &a.kv_heads, &a.head_dim, &a.win_h, &a.win_w, &a.n_edges, &f32) == 10) {
        WindowParams p;
        if (shape(&a, &p) != ESC_OK) return 1;
        const int dp = dim_padded(p.d);
        WindowParams f = p, q = p, k = p;
        show("forward", plan_forward(f, f32), f, f32, window_forward_resident(f32, dp));
        show("dq", plan_dq(q, f32), q, f32, window_dq_resident(f32, dp));
        show("dkv", plan_dkv(k, f32), k, f32, window_dkv_resident(f32, dp));
    }
}
"""


@pytest.fixture(scope="module")
def plans(lib, tmp_path_factory):  # noqa: F811
    if not os.path.exists(HIPCC):
        pytest.skip("no hipcc")
    at = tmp_path_factory.mktemp("plans")
    source, program = at / "plans.hip", at / "plans"
    source.write_text(PROGRAM)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-w", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    str(source), "-o", str(program), "-L", CSRC, "-lesc_convattn", f"-Wl,-rpath,{CSRC}"], check=True)

    def ask(cases):
        text = "\n".join(" ".join(str(int(x)) for x in c) for c in cases)
        out = subprocess.run([str(program)], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == 3 * len(cases)
        rows = [{k: v if k == "pass" else int(v) for k, v in (w.split("=") for w in line.split())} for line in out]
        return [rows[i:i + 3] for i in range(0, len(rows), 3)]
    return ask


def test_residency_is_that_of_the_built_kernels(plans):
    # a SIMD has 512 registers a lane, given out in eights
    built = {}
    for name, _, vgprs, _ in kernel_notes():
        m = re.search(r"window_(dq|dkv)_kernelI([ft])Li(\d+)E", name) or re.search(r"window_(forward)_kernelI([ft])Li(\d+)ELi1E", name)
        if m:
            key = m.group(1), m.group(2) == "f", int(m.group(3))
            built[key] = min(built.get(key, 8), 512 // ((vgprs + 7) // 8 * 8))
    assert len(built) == 3 * 2 * 3
    for (kernel, f32, dp), fits in built.items():
        row = next(r for r in plans([(1, 64, 64, 4, 4, dp, 32, 32, 0, f32)])[0] if r["pass"] == kernel)
        assert row["resident"] == fits, (kernel, f32, dp, fits)


def test_every_sharer_of_a_tiles_keys_has_keys(plans):
    # a chunk's tiles of 32 tokens are dealt to the wavefronts that share them: no more of those than tiles
    cases = [(N, H, W, heads, kv, d, *win, 0, f32)
             for N, H, W in ((1, 16, 16), (1, 64, 64), (3, 96, 96), (1, 180, 320), (5, 50, 61)) for heads, kv in ((1, 1), (4, 4), (6, 2))
             for d in (8, 16, 24, 32, 48, 64) for win in ((1, 1), (8, 8), (13, 13), (16, 16), (32, 32), (48, 48), (5, 60), (1, 300)) for f32 in (0, 1)]
    shared = 0
    for c, (r, *_) in zip(cases, plans(cases)):
        assert r["fits"] and 1 <= r["ksplit"] <= max(1, r["chunk"] // 32), (c, r)
        assert r["owners"] % r["ksplit"] == 0 and r["owners"] <= r["waves"] <= 8, (c, r)
        shared += r["ksplit"] > 1
    assert shared > 50


def test_backward_blocks_fill_the_places(plans):
    # many windows of many tiles, bf16: of the wavefronts that registers allow on a compute unit, three quarters at least are there (a block's
    # wavefronts go to the four SIMDs in turn: five to eight of them take two places of each)
    for N, H, W, heads, d, win in ((64, 64, 64, 4, 16, 32), (64, 64, 64, 4, 8, 32), (16, 96, 96, 6, 32, 48), (8, 96, 96, 6, 32, 24), (16, 64, 64, 6, 32, 32)):
        for r in plans([(N, H, W, heads, heads, d, win, win, 0, 0)])[0][1:]:
            blocks = r["resident"] // -(-r["waves"] // 4)
            assert r["fits"] and 4 * blocks * r["owners"] >= 3 * 4 * r["resident"], (N, H, W, heads, d, win, r)
