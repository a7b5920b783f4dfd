"""Which launches the linear layer's calls take, asked of the library's rules on the host (under the sanitizers): every kernel of the products is
one that the GPU tests compare with fp64, whatever the expected times of the tiles say."""
import os
import subprocess

import pytest

pytest.importorskip("torch")

import test_gpu_operators_large as large

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 20   # an aligned address; nothing is read


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("routes") / "linear_route_check")
    cmd = ["g++", "-std=c++17", "-Wall", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan",
           "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_1905_13727_amd", "csrc"),
           os.path.join(ROOT, "tests", "linear_route_check.cpp"), "-o", exe]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout

    def of(calls):
        """[launches of each call]; a call: pass, T, n, k, dtype, params, direct, and what differs from packed aligned rows"""
        lines = []
        for which, T, n, k, dtype, params, direct, *rest in calls:
            m = {**dict(x=AT, x_stride=k, dy=AT, dy_stride=n), **(rest[0] if rest else {})}
            lines.append("%s %d %d %d %d %d %d 1 %d %d %d %d" % (which, T, n, k, dtype == "bf16", params == "bf16", direct, m["x"], m["x_stride"], m["dy"], m["dy_stride"]))
        res = subprocess.run([exe], input="\n".join(lines) + "\n", stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert res.returncode == 0, res.stdout
        out = [line.split() for line in res.stdout.splitlines()]
        assert len(out) == len(calls)
        return out

    return of


def _kernels():
    sides = ("along-along", "along-across", "across-across")
    for source in ("straight", "registers", "registers-fp32", "fp32"):
        for side in sides[:2] if source == "registers-fp32" else sides:
            for tile in ("128", "64", "128/split", "64/split") + (("256",) if source == "straight" else ()):
                yield "product:%s:%s:%s" % (source, side, tile)
        for tile in ("128", "64"):
            yield "two:%s:%s" % (source, tile)
    for side in sides[:2]:
        for tile in ("256", "128"):
            yield "rest:straight:%s:%s" % (side, tile)
    yield from ("large:x", "large:w", "few", "rows", "columns", "lay:w", "lay:x", "lay:dy")


def test_every_kernel_is_tested(ask):
    taken = {t for launches in ask(large.CALLS) for t in launches}
    assert not set(_kernels()) - taken, sorted(set(_kernels()) - taken)


def test_the_graphs_hold_the_largest_tiles(ask):
    # the forward product in tiles of 256, both gradients in one launch of them, either first; rows beyond the last tile in the same launch
    f = [t for launches in ask([("f", *s, "bf16", "f32", 0) for s in large.GRAPHS]) for t in launches]
    b = [t for launches in ask([("b", *s, "bf16", "f32", 0) for s in large.GRAPHS]) for t in launches]
    assert "product:straight:along-along:256" in f and any(t.startswith("rest:") for t in f) and {"large:x", "large:w"} <= set(b), (f, b)


@pytest.mark.parametrize("n,more", [(50257, {}), (50304, dict(dy=AT + 2)), (50304, dict(dy_stride=50309))])
def test_large_gradients_that_begin_anywhere_go_straight_to_lds(ask, n, more):
    """Identity without dropout: rows of dy that do not begin on multiples of sixteen bytes (a vocabulary of odd size, a view) are laid out, as
    any dz is, and nothing else is laid out in vain."""
    for params in ("bf16", "f32"):
        for which in "bxw":
            (launches,) = ask([(which, 8192, n, 2048, "bf16", params, 1, more)])
            assert "lay:dy" in launches and not [t for t in launches if "registers" in t], launches
            assert ("lay:w" in launches) == (params == "f32" and which != "w")


def test_nothing_in_bf16_is_laid_out_for_a_product_through_registers(ask):
    """dy in place: neither weights nor input go through memory first, the products would read them through registers all the same.  fp32 weights
    do, they are rounded once."""
    (launches,) = ask([("x", 1500, 4095, 2000, "bf16", "f32", 1)])
    assert launches[0] == "lay:w" and "registers:" in launches[1]
    for which, T, n, k, params in (("x", 1500, 4095, 2001, "bf16"), ("w", 1500, 1001, 1801, "bf16"), ("b", 1500, 1001, 1801, "bf16")):
        (launches,) = ask([(which, T, n, k, "bf16", params, 1)])
        assert [t for t in launches if "registers" in t] and not [t for t in launches if t.startswith("lay")], launches
