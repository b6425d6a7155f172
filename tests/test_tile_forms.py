"""The host's rules for the tile form of a product (CPU only): the header compiled for the
host, asked for the sizes that the GPU tests and measurements name."""
import shutil
import subprocess

import pytest

from paper_2604_01622_amd import build


def ask(tmp_path, lines):
    """What `tile_forms.h` answers to C++ expressions of an integer or enumeration."""
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("needs g++")
    src, exe = tmp_path / "forms.cpp", tmp_path / "forms"
    body = "\n".join(f'  std::printf("%d\\n", static_cast<int>({x}));' for x in lines)
    src.write_text('#include <cstdio>\n#include "tile_forms.h"\nusing namespace ec;\n'
                   f"int main() {{\n{body}\n}}\n")
    subprocess.run([cc, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", build.CSRC, str(src), "-o",
                    str(exe)], check=True, capture_output=True, text=True)
    r = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60)
    return [int(x) for x in r.stdout.split()]


SMALL, WIDE, BIG = range(3)


def test_fp32_weight_gradients_of_packed_rows(tmp_path):
    """64 x 128 tiles up to one round of them, 128 x 128 past it, never 64 x 64."""
    sizes = [  # experts, d, h, the forms of dW2 [d, h] and dW1/dW3 [2 h, d]
        (17, 512, 512, WIDE, BIG),      # 544 and 1088 tiles of 64 x 128
        (24, 512, 512, WIDE, BIG),      # 768: one whole round
        (12, 512, 512, WIDE, WIDE),     # 384 and 768
        (13, 512, 512, WIDE, BIG),      # 416 and 832
        (20, 640, 512, BIG, BIG),       # 800
        (16, 1024, 512, BIG, BIG),      # the small model of the listed cases
        (130, 256, 256, BIG, BIG),
        (3, 256, 256, WIDE, WIDE),
        (1, 64, 64, WIDE, WIDE),
    ]
    lines = []
    for E, d, h, _, _ in sizes:
        lines += [f"f32_form(F32Rows::PACKED_K, {E}, {d}, {h})",
                  f"f32_form(F32Rows::PACKED_K, {E}, {2 * h}, {d})"]
    assert ask(tmp_path, lines) == [f for s in sizes for f in s[3:]]


def test_fp32_products_of_rows(tmp_path):
    """Packed rows take 64 x 128 tiles; uniform batches 128 x 128 from one per CU on."""
    lines = ["f32_form(F32Rows::PACKED, 1, 1, 64)", "f32_form(F32Rows::PACKED, 256, 9000, 4096)",
             "f32_form(F32Rows::UNIFORM, 255, 128, 128)", "f32_form(F32Rows::UNIFORM, 256, 128, 128)",
             "f32_form(F32Rows::UNIFORM, 64, 129, 129)"]
    assert ask(tmp_path, lines) == [WIDE, WIDE, SMALL, BIG, BIG]
