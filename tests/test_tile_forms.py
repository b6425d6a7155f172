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


# Tiles (rows, columns) of a training step's bf16 products.
T256, T192, T128, SQ = (256, 256), (192, 256), (128, 256), (128, 128)
HALF_DW2, HALF_DW13 = (256, 128), (128, 256)
BF16_FORMS = [
    # tokens, d, experts, h, top k, shared width; W1/W3, W2, dA, dX, dW2, dW1/dW3; those of the
    # shared experts' W1/W3, W2, dA, dX
    ((700, 768, 4, 640, 2, 256), (SQ, SQ, SQ, SQ, HALF_DW2, HALF_DW13), (SQ, SQ, SQ, SQ)),
    ((700, 64, 32, 512, 4, 0), (T128, SQ, SQ, SQ, HALF_DW2, HALF_DW13), ()),
    ((700, 64, 48, 512, 8, 0), (T192, SQ, SQ, SQ, HALF_DW2, HALF_DW13), ()),
    ((4000, 64, 48, 512, 2, 0), (T256, SQ, SQ, SQ, HALF_DW2, HALF_DW13), ()),
    ((700, 1024, 32, 64, 4, 0), (SQ, T128, SQ, SQ, HALF_DW2, HALF_DW13), ()),
    ((700, 1024, 48, 64, 8, 0), (SQ, T192, SQ, T256, HALF_DW2, HALF_DW13), ()),
    ((4000, 1024, 48, 64, 2, 640), (SQ, T256, SQ, T256, HALF_DW2, HALF_DW13), (T128, SQ, SQ, SQ)),
    ((2500, 64, 48, 768, 4, 0), (T128, SQ, T256, SQ, HALF_DW2, T256), ()),
    ((200, 64, 130, 64, 2, 0), (T256, T256, T256, T256, HALF_DW2, HALF_DW13), ()),
    ((900, 256, 130, 256, 8, 0), (T256, T256, T256, T256, HALF_DW2, T256), ()),
    ((10000, 64, 200, 64, 8, 0), (SQ, SQ, SQ, SQ, T256, HALF_DW13), ()),
    ((26000, 256, 2, 64, 1, 64), (SQ, T128, SQ, SQ, HALF_DW2, HALF_DW13), (SQ, T128, SQ, SQ)),
    ((40000, 256, 2, 128, 1, 128), (T192, T192, SQ, T256, HALF_DW2, HALF_DW13),
     (T192, T192, SQ, T256)),
    ((60000, 256, 2, 128, 1, 256), (T256, T256, SQ, T256, HALF_DW2, HALF_DW13),
     (T256, T256, T256, T256)),
]


def test_bf16_training_products(tmp_path):
    """Every form that a product has is taken at some of these sizes, as written there."""
    lines, want = [], []
    for (n, d, E, h, k, hs), packed, shared in BF16_FORMS:
        for rows, width, tiles in ((f"RowsOf{{true, {E}, {n * k}}}", h, packed),
                                   (f"RowsOf{{false, 1, {n}}}", hs, shared)):
            if tiles:
                lines += [f"fwd_rows_form({rows}, {2 * width})", f"fwd_rows_form({rows}, {d})",
                          f"bwd_rows_half({rows}, {width}, true)",
                          f"bwd_rows_half({rows}, {d}, false)"]
                want += tiles[:4]
        lines += [f"dW2_half_wide({E}, {n * k}, {d}, {h})", f"dW13_half_wide({E}, {n * k}, {d}, {h})"]
        want += packed[4:]
    got = []
    for line, answer in zip(lines, ask(tmp_path, lines)):
        forms = {"fwd_rows_form": (T256, T192, T128, SQ), "bwd_rows_half": (T256, SQ),
                 "dW2_half_wide": (T256, HALF_DW2), "dW13_half_wide": (T256, HALF_DW13)}
        got.append(forms[line[:line.index("(")]][answer])
    assert got == want
    for column, forms in enumerate([{T256, T192, T128, SQ}] * 2 + [{T256, SQ}] * 2
                                   + [{T256, HALF_DW2}, {T256, HALF_DW13}]):
        assert {p[column] for _, p, _ in BF16_FORMS} == forms
    for column, forms in enumerate([{T256, T192, T128, SQ}] * 2 + [{T256, SQ}] * 2):
        assert {s[column] for _, _, s in BF16_FORMS if s} == forms
