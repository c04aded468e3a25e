"""The tiles that the cases of the GPU tests run on, asked of the library on the
host: a changed estimate must not move a test off the kernel it is for."""

import re
import subprocess

import paper_1911_07384_amd as F
import test_gpu_int8 as int8
import test_gpu_muon as muon

def test_every_tile_of_the_products_is_covered():
    """A, B and X', with one product and with three, on every tile that the rule ever
    gives them; reductions in parts are offered to A only."""
    for products in (1, 3):
        seen = [set(), set(), set()]
        for shapes in muon.SETS:
            kinds = F.fp16_muon_kernels(F.muon_descs(shapes), products).split(", ")
            for s, k in zip(seen, kinds):
                s.add("parts" if " in " in k else k)
        plain = {"256", "192", "128", "128 deep", "64"}
        assert seen[0] == plain | {"64 deep", "parts"}, (products, seen[0])
        assert seen[1] == plain | ({"64 deep"} if products == 3 else set()), (products, seen[1])
        assert seen[2] == plain | ({"64 deep"} if products == 3 else set()), (products, seen[2])


def test_small_sets_take_one_workgroup_each():
    name = lambda *shapes: F.fp16_muon_kernels(F.muon_descs(list(shapes)), 1)
    small = "one workgroup each"
    assert name((64, 1024)) == name((1024, 64)) == name(*[(64, 576)] * 24) == small
    assert small not in (name((65, 65)), name((64, 1025)), name(*[(8, 8)] * 25),
                         name((64, 64), (128, 128)))


def test_every_tile_of_the_8_bit_product_is_covered():
    got = {F.fp16_int8_kernel(*c) for c in int8.PRODUCTS}
    assert F.fp16_int8_kernel(16, 8192, 300) == "few rows" != F.fp16_int8_kernel(16, 8193, 300)
    assert got == {"few rows", "tile 64", "tile 128", "tile 128 deep", "tile 256"}


def test_no_tile_is_built_that_no_product_runs_on():
    """The kernels of A and B (one each for a tile and a number of products) and of X'
    (two: the last step's stores differ) in the library are those that the sets above
    reach, so that every one of them runs in a GPU test."""
    symbols = subprocess.run(["nm", "-C", F.LIB_PATH], capture_output=True, text=True, check=True).stdout
    for products in (1, 3):
        seen = [set(), set(), set()]
        for shapes in muon.SETS:
            for s, k in zip(seen, F.fp16_muon_kernels(F.muon_descs(shapes), products).split(", ")):
                s.add(k if " in " not in k else "parts")
        a, b, x = (len(s - {"parts"}) for s in seen)
        built = lambda kernel, tail: len(re.findall(rf"__device_stub__{kernel}<.*>, {tail}>\(", symbols))
        assert built("ns_sym", f"0, {products}") == a, products
        assert built("ns_sym", f"1, {products}") == b, products
        for last in ("false", "true"):
            assert built("ns_x", f"{products}, {last}") == x, products
