"""The rules that choose the kernel of an 8-bit product (csrc/int8_route.cpp: plain host C++) without a GPU, and that the GPU tests reach every
kernel at its edges: a threshold that moves must not take a test's kernel away unseen."""
import os
import shutil
import subprocess

import pytest

import test_gpu_int8_routes as routes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_12357_amd", "csrc")
CUS = 256
TILES = ["k64Shared", "k64", "k64Short", "k128Shared", "k128"]
HEIGHT = {"wide2": 128, "wide3": 192, "wide4": 256}      # tokens of a tile; 64 of the others
WIDTH = {"k64Shared": 64, "k64": 64, "k64Short": 64, "k128Shared": 128, "k128": 128}


@pytest.fixture(scope="module")
def route(tmp_path_factory):
    cxx = shutil.which(os.environ.get("CXX", "g++"))
    if cxx is None:
        pytest.skip("no host C++ compiler")
    out = str(tmp_path_factory.mktemp("route") / "int8_route_check")
    subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-static-libasan", "-static-libubsan", "-Wall", "-Wextra", "-Werror", "-I", CSRC,
                    os.path.join(ROOT, "tests", "host", "int8_route_check.cpp"), os.path.join(CSRC, "int8_route.cpp"), "-o", out], check=True)
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0")
    env.pop("LD_PRELOAD", None)

    def ask(sizes):
        """-> a kernel's name for each (T, N, K)."""
        r = subprocess.run([out], input="".join(f"{t} {n} {k} {CUS}\n" for t, n, k in sizes), capture_output=True, text=True, check=True, env=env)
        names = []
        for line in r.stdout.splitlines():
            streams, ask.fused, blocks, tile = map(int, line.split())
            names.append("stream" if streams else f"wide{blocks}" if blocks else TILES[tile])
        assert len(names) == len(sizes)
        return names
    return ask


def test_sizes_are_listed_under_the_kernel_that_they_take(route):
    for name, sizes in routes.ROUTES.items():
        assert route(sizes) == [name] * len(sizes), name
    assert set(routes.ROUTES) == set(HEIGHT) | set(TILES)


@pytest.mark.parametrize("name", routes.ROUTES)
def test_every_kernel_has_its_edges(name):
    """A kernel that no size of K below 13 chunks takes has none of a vector or three chunks."""
    sizes, h, w = routes.ROUTES[name], HEIGHT.get(name, 64), WIDTH.get(name, 256)
    short = not name.endswith("Shared")
    seen = [("rest", k % 16 > 0) for _, _, k in sizes] + [("no vector", k < 16) for _, _, k in sizes] + [("chunk in part", k % 128 > 0) for _, _, k in sizes]
    seen += [("below three chunks", 16 < k < 384 and k % 16 > 0) for _, _, k in sizes] + [("ragged tokens", t % h > 0) for t, _, _ in sizes]
    seen += [("ragged outputs", n % w > 0) for _, n, _ in sizes] + [("whole", t % h == n % w == k % 128 == 0) for t, n, k in sizes]
    seen += [("one output in the last tile", n % w == 1) for _, n, _ in sizes] + [("one token in the last tile", t % h == 1) for t, _, _ in sizes]
    seen += [("vectors, no rest", k % 16 == 0 and k % 128 > 0) for _, _, k in sizes] + [("tiles of one workgroup", -(-t // h) * -(-n // w) > CUS) for t, n, _ in sizes]
    seen = {what for what, there in seen if there}
    want = {"rest", "chunk in part", "ragged tokens", "ragged outputs", "whole"}
    if short:
        want |= {"no vector", "below three chunks"}
    if name in HEIGHT:
        want |= {"tiles of one workgroup", "vectors, no rest"}
    assert want <= seen, want - seen


def test_parts_of_one_product_take_every_kernel(route):
    for K, parts in routes.PARTS.items():
        assert all(0 <= t0 < t1 <= routes.WHOLE[0] and 0 <= n0 < n1 <= routes.WHOLE[1] for t0, t1, n0, n1 in parts)
    on = {K: set(route([(t1 - t0, n1 - n0, K) for t0, t1, n0, n1 in parts])) for K, parts in routes.PARTS.items()}
    assert on[1723] | on[601] == set(HEIGHT) | set(TILES) | {"stream"}
    assert len(on[1723]) >= 7 and len(on[601]) >= 4


def test_up_to_64_tokens_stream_while_their_codes_fit(route):
    for T, K in ((1, 16384), (16, 16384), (17, 8192), (32, 8192), (33, 4096), (64, 4096)):
        assert route([(T, 1000, K), (T, 1000, K + 1)])[0] == "stream" and route([(T, 1000, K + 1)])[0] != "stream"
    assert route([(65, 1000, 64)])[0] != "stream"


def test_small_batches_are_quantised_by_the_product(route):
    for T, K in ((1, 16384), (2, 8192), (8, 2048), (16, 1024)):
        assert route([(T, 100, K)]) and route.fused == 1
        assert route([(T, 100, K + 1)]) and route.fused == 0
    assert route([(17, 100, 10)]) and route.fused == 0
