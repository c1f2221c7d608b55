"""Which kernels and shapes a call on 8-bit experts takes (csrc/fp8_forms.h), asked on the host."""
import os
import shutil
import subprocess

import pytest

from paper_2503_05066_amd import build, capmoe

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = "/opt/rocm/include"
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(ROCM), reason="g++ and the HIP headers are needed")

HARNESS = r"""
#include <stdio.h>
#include <string>
#include "fp8_forms.h"
using namespace capmoe;
static std::string tiles(const Fp8Gemm& g, bool gate_up, int cus) {
    const int columns = gate_up ? 128 : (fp8_tiles_are_wide(g, cus) ? 256 : 128);
    return std::to_string(columns) + "x" + std::to_string(1 << fp8_tile_shift(g.max_rows, g.experts, g.n_pad / columns, cus));
}
static std::string few(const Fp8Gemm& g, bool gate_up, int cus) {
    const int cols = gate_up ? 16 : 32;
    const int64_t waves = std::min<int64_t>(g.max_rows, g.experts) * ((g.n + cols - 1) / cols);
    return "few/" + std::to_string(fp8_thin_split(waves, g.pitch / kFp8Block, cus));
}
int main() {
    char what;
    int a, e, k, d, h, mode, cus;
    double gamma;
    while (scanf(" %c %d", &what, &cus) == 2) {
        if (what == 'p') {  // a product: rows, experts, columns of x, columns of y
            if (scanf("%d %d %d %d", &a, &e, &d, &h) != 4) return 1;
            const Fp8Gemm g = fp8_gemm(e, a, d, h);
            printf("%s%s\n", (fp8_gemm_is_few_rows(g) ? few(g, false, cus) : tiles(g, false, cus)).c_str(),
                   fp8_weights_stream((double)g.experts * g.pitch * g.n_pad) ? " stream" : "");
        } else {            // an FFN: tokens, experts, top-k, d, h, mode, gamma
            if (scanf("%d %d %d %d %d %d %lf", &a, &e, &k, &d, &h, &mode, &gamma) != 7) return 1;
            moe_desc_t desc{};
            desc.n_tokens = a, desc.d_model = d, desc.n_experts = e, desc.top_k = k, desc.d_hidden = h, desc.device_groups = 1;
            desc.mode = mode, desc.capacity_scope = 1, desc.gamma = gamma, desc.dtype = MOE_DTYPE_BF16;
            if (validate(&desc) != MOE_OK) { puts("refused"); continue; }
            const Sizes s = derive(desc);
            const Fp8Gemm up = fp8_gemm(e, s.max_rows, d, fp8_pitch(h)), down = fp8_gemm(e, s.max_rows, fp8_pitch(h), d);
            const bool f = fp8_ffn_is_few_rows(desc, s);
            printf("%s %s%s\n", (f ? few(up, true, cus) : tiles(up, true, cus)).c_str(), (f ? few(down, false, cus) : tiles(down, false, cus)).c_str(),
                   fp8_weights_stream(3.0 * e * up.pitch * up.n_pad) ? " stream" : "");
        }
    }
}
"""

NONE = capmoe.MODE_NONE
PRODUCTS = [  # rows, experts, columns of x, columns of y -> on 256, 128 and 32 compute units
    ((8, 64, 2048, 1024), ("few/4", "few/4", "few/1")),
    ((128, 64, 2048, 1024), ("few/1", "few/1", "few/1")),
    ((203, 1, 2056, 5640), ("128x64", "128x128", "128x256")),  # 45 column blocks: 180 items of 64 rows, 90 of 128
    ((1024, 1, 2056, 5640), ("128x256",) * 3),
    ((1024, 8, 4096, 14336), ("256x256 stream",) * 3),
    ((1024, 8, 14336, 4096), ("128x256 stream", "256x256 stream", "256x256 stream")),
    ((32768, 64, 2048, 1024), ("256x256",) * 3),
    ((16384, 8, 14336, 4096), ("256x256 stream",) * 3),
    ((20000, 12, 256, 120), ("128x128", "128x256", "128x256")),
]
FFNS = [  # tokens, experts, top-k, d, h
    ((1, 64, 8, 2048, 1024), ("few/4 few/4 stream", "few/2 few/2 stream", "few/1 few/1 stream")),
    ((16, 8, 2, 4096, 14336), ("few/1 few/4 stream", "few/1 few/1 stream", "few/1 few/1 stream")),
    ((512, 8, 2, 2048, 1024), ("128x64 128x128", "128x128 128x256", "128x256 256x256")),
    ((4096, 64, 8, 2048, 1024), ("128x256 256x256 stream",) * 3),
]
UNITS = (256, 128, 32)


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    folder = tmp_path_factory.mktemp("forms")
    (folder / "main.cpp").write_text(HARNESS)
    capmoe.load()
    subprocess.run(["g++", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", ROCM, "-I", os.path.join(ROOT, "include"), "-I", build.CSRC,
                    str(folder / "main.cpp"), "-o", str(folder / "main"), build.LIB, "-Wl,-rpath," + os.path.dirname(build.LIB),
                    "-Wl,--allow-shlib-undefined"], check=True)

    def call(kind, cus, sizes, mode=NONE, gamma=1.0):
        text = f"{kind} {cus} " + " ".join(map(str, sizes)) + ("" if kind == "p" else f" {mode} {gamma}")
        return subprocess.run([str(folder / "main")], input=text, capture_output=True, text=True, check=True).stdout.strip()

    return call


@pytest.mark.parametrize("sizes,forms", PRODUCTS, ids=lambda v: "-".join(map(str, v)) if isinstance(v[0], int) else "")
def test_forms_of_a_product_follow_the_compute_units(ask, sizes, forms):
    assert tuple(ask("p", cus, sizes) for cus in UNITS) == forms


@pytest.mark.parametrize("sizes,forms", FFNS, ids=lambda v: "-".join(map(str, v)) if isinstance(v[0], int) else "")
def test_forms_of_an_ffn_follow_the_compute_units(ask, sizes, forms):
    assert tuple(ask("f", cus, sizes) for cus in UNITS) == forms


# An expert may have all rows of a product, and a row of every token in an FFN: at most four passes over its weights, 32 and 16 rows each.
@pytest.mark.parametrize("e,k,n", [(256, 512, 512), (64, 2048, 1024), (60, 512, 1280), (128, 2048, 768)])
def test_products_whose_rows_may_lie_on_one_expert(ask, e, k, n):
    assert ask("p", 256, (128, e, k, n)).startswith("few")
    for rows in (129, 512, 8 * e, 32 * e):
        assert ask("p", 256, (rows, e, k, n))[:3] in ("128", "256")


@pytest.mark.parametrize("e,top_k,d,h", [(256, 8, 256, 256), (128, 4, 2048, 768), (64, 4, 2048, 1024), (64, 8, 512, 512)])
def test_ffns_whose_tokens_may_lie_on_the_same_experts(ask, e, top_k, d, h):
    assert ask("f", 256, (64, e, top_k, d, h)).startswith("few")
    for tokens in (65, 128, 512):
        assert ask("f", 256, (tokens, e, top_k, d, h))[:3] in ("128", "256")
    # a capacity bounds them too: one pass, and four
    tokens = 16 * e // top_k
    assert ask("f", 256, (tokens, e, top_k, d, h), capmoe.MODE_TOKEN_DROP, 1.0).startswith("few")
    assert ask("f", 256, (tokens, e, top_k, d, h), capmoe.MODE_TOKEN_DROP, 4.0).startswith("few") == (3 * e * d * h <= 64 << 20)


def test_gpu_cases_have_the_forms_that_they_name(ask):
    import test_gpu_fp8 as on_gpu

    for counts, k, n, form in on_gpu.PRODUCT_FORMS + on_gpu.STREAMED_PRODUCTS:
        assert ask("p", 256, (sum(counts), len(counts), k, n)) == form, (counts, k, n)
    for tokens, k, counts, d, h, forms in on_gpu.STREAMED_FFNS:
        assert ask("f", 256, (tokens, len(counts), k, d, h)) == forms, (tokens, d, h)
