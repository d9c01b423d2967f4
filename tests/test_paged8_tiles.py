"""CPU run of the index arithmetic of the matrix kernels over a cache of 8 bits, as tests/test_paged_tiles.py runs that of the others: their tiles and
groups of keys, and the scales that they read for a group."""
import os
import subprocess

from tests.test_paged_tiles import ROOT, TILES

# (of a group that is there, the scales of all of its blocks are read, behind the last key too: they are the page's)
SCALES = r"""
    const int blocks = (1 << c.shift) / 16, first = (key & ((1 << c.shift) - 1)) / 16;
    if (first < 0 || first + size / 16 > blocks) return fail("scales outside the page's", key, size, blocks);
    return 0;
}

// All tiles"""
RUNS = r"""
        // bf16: tiles of 128 and of 32 rows, fp32: of 16; groups of 16 keys, or of 32 or 64 in pages that hold them
        if (run<128, 64>(c, 16) || run<32, 64>(c, 16) || run<16, 64>(c, 16)) return 1;
        if (c.shift >= 5 && (run<32, 64>(c, 32) || run<16, 64>(c, 32))) return 1;
        if (c.shift >= 6 && (run<128, 64>(c, 64) || run<32, 64>(c, 64) || run<16, 64>(c, 64))) return 1;
    }
    return 0;
}
"""


def test_no_read_of_the_matrix_kernels_leaves_the_pages_and_their_scales(tmp_path):
    code, end = TILES[:TILES.index("        // bf16:")] + RUNS, "    return 0;\n}\n\n// All tiles"
    assert code.count(end) == 1
    src = tmp_path / "tiles8.cpp"
    src.write_text(code.replace(end, SCALES))
    exe = str(tmp_path / "tiles8")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined,address", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2503_02356_amd", "csrc"), str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr[-2000:]
