"""Where the pieces of a row tile's steps begin and end, as the attention kernel
computes it, for lengths up to the largest that is taken.  No GPU: the header's
function is compiled for the host."""
import importlib.util
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <cstdio>
#include "heads.h"
int main() {
    int n, parts;
    while (scanf("%d %d", &n, &parts) == 2)
        for (int i = 0; i <= parts; ++i) printf("%d ", caee::head_piece_at(n, i, parts));
}
"""


@pytest.fixture(scope="module")
def piece_at(tmp_path_factory):
    spec = importlib.util.spec_from_file_location("caee_build", os.path.join(ROOT, "paper_2606_29982_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    at = tmp_path_factory.mktemp("pieces")
    (at / "pieces.hip").write_text(SOURCE)
    subprocess.run([build.hipcc(), "-std=c++17", "-O1", "--cuda-host-only", "-I", build.CSRC, "-c", str(at / "pieces.hip"),
                    "-o", str(at / "pieces.o")], check=True)
    subprocess.run([build.hipcc(), str(at / "pieces.o"), "-o", str(at / "pieces")], check=True)

    def run(cases):
        out = subprocess.run([str(at / "pieces")], input="\n".join(f"{n} {p}" for n, p in cases), capture_output=True,
                             text=True, check=True)
        return [int(x) for x in out.stdout.split()]
    return run


def test_pieces_cover_the_steps_at_every_length(piece_at):
    """64 tokens a step, 2^30 tokens at most; up to 64 pieces of one of 64 requests, up to 1024 of one of more."""
    cases = [(n, p) for n in (0, 1, 2, 63, 64, 65, 1000, 1563, 2 ** 20 + 1, 2 ** 22 - 1, 2 ** 22, 2 ** 22 + 1, 2 ** 23,
                              2 ** 24 - 1, 2 ** 24) for p in (1, 2, 3, 63, 64, 65, 256, 511, 512, 513, 1023, 1024)]
    want = [n * i // p for n, p in cases for i in range(p + 1)]
    assert piece_at(cases) == want
