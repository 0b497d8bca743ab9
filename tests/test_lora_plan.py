"""How the adapters' kernels divide their work, asked of the library's own rules (gm_lora.h, compiled for the host)."""
import os
import shutil
import subprocess

import pytest

import test_gpu_lora_lengths as lengths
import test_gpu_lora_wide_blocks as wide

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("lora") / "lora_plan")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-o", exe, os.path.join(HERE, "lora_plan.cpp")], check=True)

    def ask(op, shapes):  # (T, n, d_in, widths, r)
        text = "".join(f"{op} {T} {n} {d} {r} {len(w)} {' '.join(map(str, w))}\n" for T, n, d, w, r in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(shapes)
        return out

    return ask


def test_forward_blocks_beyond_64_ranks_by_what_runs_at_once(plan):
    # one block per CU there (99 KB of LDS): the widths that were measured best, with 256, 512 and 1024 columns tried
    best = [(2048, 1, 512, (4096,), 128, 512), (1024, 1, 512, (11008,), 128, 1024), (4096, 1, 512, (4096,), 72, 1024),
            (512, 1, 512, (4096,), 128, 256), (64, 32, 512, (4096,), 128, 512), (8192, 1, 512, (11008,), 128, 1024),
            (203, 40, 512, (4096,) * 3, 96, 1024), (2048, 1, 512, (4096,), 64, 256), (1024, 1, 512, (11008,), 64, 256)]
    assert [int(g.split("/")[0]) for g in plan("fwd", [b[:5] for b in best])] == [b[5] for b in best]


def test_dx_of_more_than_128_ranks_takes_the_columns_in_lds(plan):
    assert plan("dx", [(4096, 1, 8192, (64,) * 4, 128), (64, 40, 64, (64,) * 3, 64)]) == ["256/256"] * 2


def test_gradient_lengths(plan):
    # what the GPU tests' shapes are named to take
    shapes = [(sum(counts) + none, n, d, w, r) for counts, n, d, w, r, none, _ in lengths.LENGTHS]
    assert [int(g) for g in plan("length", shapes)] == [x[6] for x in lengths.LENGTHS]
    assert {x[6] for x in lengths.LENGTHS} == {512, 1024, 2048}
    for length in (512, 1024, 2048):
        counts = [k for x in lengths.LENGTHS if x[6] == length for k in x[0]]
        assert any(k > length for k in counts) and any(k == length or k % length == 1 for k in counts)
        assert any(k < length for k in counts)


def test_widths_of_blocks(plan):
    shapes = [(sum(wide.TILES) + 3, 40, d, w, r) for d, w, r, _, _ in wide.WIDE]
    fwd, dx = ([tuple(map(int, g.split("/"))) for g in plan(op, shapes)] for op in ("fwd", "dx"))
    assert [g[0] for g in fwd] == [x[3] for x in wide.WIDE] and [g[0] for g in dx] == [x[4] for x in wide.WIDE]
    # every number of rank blocks (16, 32, 64, 128 ranks) has a block, of a part that is as wide, with weights loaded anew
    anew = {(op, -(-ranks // 16)) for x, f, b in zip(wide.WIDE, fwd, dx)
            for op, ranks, got, widest in (("fwd", x[2], f, max(x[1])), ("dx", x[2] * len(x[1]), b, x[0]))
            if got[0] > got[1] and widest > got[1]}
    for op in ("fwd", "dx"):
        blocks = {b for o, b in anew if o == op}
        assert 1 in blocks and 2 in blocks and blocks & {3, 4} and blocks & {5, 6, 7, 8}, (op, blocks)
