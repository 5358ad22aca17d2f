"""Which products in 16 bits go to blocks of 32 rows of w by 64 tokens, without a GPU: those of short rows whose results do not leave tiles straight from registers, up to a block a compute unit."""
import subprocess

import pytest

import dispatch
from test_product_choice import SOURCE


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("product")
    source = SOURCE.replace("words, exact8;", "words, exact8, direct;").replace('"%d %d %d %d %d %d %d %d"', '"%d %d %d %d %d %d %d %d %d"').replace("&exact8) == 8", "&exact8, &direct) == 9")
    (d / "choice.cpp").write_text(source.replace("bits, words, exact8);", "bits, words, exact8, direct);"))
    dispatch.compile_host(["-o", str(d / "choice"), str(d / "choice.cpp")])

    def run(n, k, cols, gated=0, to8=0, direct=0):
        text = "%d %d %d %d %d 16 1 0 %d\n" % (n, 2 * k, cols, gated, to8, direct)
        return int(subprocess.run([str(d / "choice")], input=text, capture_output=True, text=True, check=True).stdout.split()[0])
    return run


def test_short_rows_that_leave_through_lds(ask):
    for n, k, cols, gated in ((308, 1160, 1100, 0), (400, 1280, 1004, 0), (1000, 904, 470, 0), (100, 1160, 2500, 0), (700, 1160, 700, 0), (308, 1160, 550, 1), (40, 1000, 7000, 0)):
        assert ask(n, k, cols, gated) == 24 and ask(n, k, cols, gated, direct=1) == 3, (n, k, cols)
    for n, k, cols in ((308, 1288, 1100), (700, 1536, 700), (600, 1000, 1300), (1000, 512, 1004)):          # longer rows, more blocks
        assert ask(n, k, cols) in (3, 4), (n, k, cols)
    assert ask(64, 4096, 4096) == 22 and ask(308, 1160, 544, gated=1, to8=1) != 24
