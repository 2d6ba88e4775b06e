"""Which kernels the entry points around a gated memory launch, by sizes and layouts, found on the CPU: a small program takes the place of the runtime's launch
and prints what it is asked for (host_launches/memory_launches.cpp).  What a rule chooses has no part in a call's results, so that no other test sees it."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PACKAGE = os.path.join(ROOT, "paper_2509_10771_amd")
CLANGXX = os.environ.get("CLANGXX", "/opt/rocm/lib/llvm/bin/clang++")
F32, BF16, F16 = 0, 1, 2

pytestmark = pytest.mark.skipif(not os.path.exists(CLANGXX), reason="clang++ not installed")


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """launches(call) -> [(kernel, its template's arguments, workgroups)]."""
    exe = str(tmp_path_factory.mktemp("launches") / "memory_launches")
    subprocess.run([CLANGXX, "-std=c++17", "-O1", os.path.join(ROOT, "tests", "host_launches", "memory_launches.cpp"), "-o", exe,
                    os.path.join(PACKAGE, "librslx.so"), "-Wl,-rpath," + PACKAGE, "-Wl,--export-dynamic", "-Wl,--allow-shlib-undefined"], check=True)

    def ask(call):
        out = subprocess.run([exe], input=call + "\n", capture_output=True, text=True, check=True, timeout=60).stdout
        found = re.findall(r"(\w+)(?:<([^;]*)>)? (\d+)x\d+; ", out)
        assert found, (call, out)
        return [(kernel, tuple(arguments.split(", ")), int(groups)) for kernel, arguments, groups in found]
    return ask


def _side_by_side(kind, dtype, T, N, D):
    """Candidates and gates side by side [T, N, 2 D], as one product leaves them; everything else [T, N, D]."""
    return "%s %d %d %d %d %d %d %d %d" % (kind, dtype, T, N, D, 2 * N * D, 2 * D, N * D, D)


def _by_sequence(kind, dtype, T, N, D):
    """The same with a sequence's steps one after another [N, T, ..]."""
    return "%s %d %d %d %d %d %d %d %d" % (kind, dtype, T, N, D, 2 * D, 2 * T * D, D, T * D)


def _whole(found):
    """Whether all walks and steps of a call take rows as whole, aligned loads."""
    walks = [arguments for kernel, arguments, _ in found if kernel.startswith("recurrence") and "join" not in kernel]
    assert walks
    return all("true" == arguments[1 if len(arguments) == 2 else 3] for arguments in walks)


@pytest.mark.parametrize("dtype,T,N,D", [(F32, 24, 4096, 256), (F32, 24, 8192, 256), (F32, 24, 4096, 512), (BF16, 24, 16384, 256), (F16, 20, 16384, 256),
                                         (F32, 24, 16384, 512), (F32, 2, 65536, 1024), (BF16, 100, 8192, 512), (F32, 300, 4096, 256)])
@pytest.mark.parametrize("kind", ["forward", "backward"])
def test_many_aligned_environments_are_whole_loads(launches, kind, dtype, T, N, D):
    """Steps of many environments lie far apart; what has to fit 32 bits is the steps that one workgroup holds, of those that there are."""
    for layout in (_side_by_side, _by_sequence):
        assert _whole(launches(layout(kind, dtype, T, N, D)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N", [64, 8192, 16384, 1 << 20])
def test_one_step_has_no_distance(launches, dtype, N):
    """The distance of steps is not used where there is one, whatever it is."""
    D = 256
    for step in (2 * N * D, 0, 7, -3, 1 << 40, -(1 << 62)):
        for kind in ("step", "forward", "backward"):
            assert _whole(launches("%s %d 1 %d %d %d %d %d %d" % (kind, dtype, N, D, step, 2 * D, step, D)))


@pytest.mark.parametrize("kind,T,N,D,step", [("forward", 24, 8, 256, 1 << 40), ("backward", 24, 8, 256, 1 << 25), ("forward", 24, 8, 256, -4096), ("forward", 24, 8, 256, 4099),
                                             ("backward", 24, 8, 255, 4096), ("step", 1, 8, 255, 0)])
def test_rows_that_start_anywhere_or_far_apart_are_not(launches, kind, T, N, D, step):
    assert not _whole(launches("%s %d %d %d %d %d %d %d %d" % (kind, F32, T, N, D, step, 2 * D, N * D, D)))


@pytest.mark.parametrize("dtype,T,N,D", [(BF16, 32, 12288, 256), (F16, 32, 12288, 256), (BF16, 24, 16384, 256), (F32, 24, 8192, 256), (F32, 20, 4096, 512)])
def test_large_roll_outs_go_past_the_caches(launches, dtype, T, N, D):
    """The calls of test_gpu_memory_paths.py: one walk, which reads and writes past the caches."""
    for kind, kernel, steps in (("forward", "recurrence_kernel", "4"), ("backward", "recurrence_backward_kernel", "8")):
        (name, arguments, _), = launches(_side_by_side(kind, dtype, T, N, D))
        assert name == kernel and arguments[1:] == (steps, "1", "true", "2", "false")


def _symmetric(found):
    """The kernels of X X^T and its square, each once, with their workgroups."""
    return sorted({(kernel, arguments[0], groups) for kernel, arguments, groups in found if arguments[0] in ("(MuonProduct)0", "(MuonProduct)1")})


@pytest.mark.parametrize("shapes,large", [
    ("1536x1536", False), ("1800x1800", False), ("1930x1930", False), ("2048x4096", True), ("4096x2048", True), ("2048x8192", True), ("2176x2176", True), ("2304x2304", False),
    ("2600x2600", True), ("2700x2700", False), ("3000x3000", False), ("3456x3456", True), ("3500x3500", True), ("4096x4096", False),
    (",".join(["1024x1024"] * 4), False), (",".join(["1000x1024"] * 10), False), (",".join(["600x610"] * 32), False), ("512x256,256x128,128x12", False)])
def test_symmetric_products_take_large_tiles_where_these_gain(launches, shapes, large):
    """Both sides of these were timed; two rounds over the compute units for a few tiles more than there are of those, or short contractions in pieces, lose."""
    kernels = {kernel for kernel, _, _ in _symmetric(launches("muon " + shapes))}
    assert kernels == ({"muon_large_kernel", "muon_fold_kernel"} if large else {"muon_product_kernel"})


@pytest.mark.parametrize("large", ["2048x4096", "4096x2048", "3500x3500", "2600x2600,2600x2700"])
@pytest.mark.parametrize("small", ["30x100", "2048x12", "512x2048", "12x12,1x1", "480x65536", "1000x1000,300x200"])
def test_a_small_matrix_takes_nothing_from_a_large_one(launches, large, small):
    """Symmetric products of large matrices in large tiles and pieces of the contraction, whatever else is in the call, and wherever: the same workgroups, or more
    of the same round where smaller matrices go with them."""
    alone, beside = _symmetric(launches("muon " + large)), small.split(",")
    assert [kernel for kernel, _, _ in alone] == ["muon_fold_kernel"] * 2 + ["muon_large_kernel"] * 2
    for together in (large.split(",") + beside, beside + large.split(","), large.split(",")[:1] + beside + large.split(",")[1:]):
        found = _symmetric(launches("muon " + ",".join(together)))
        there = [x for x in found if x[0] != "muon_product_kernel"]
        assert there == alone or ([x[:2] for x in there] == [x[:2] for x in alone] and all(a[2] < b[2] <= max(256, a[2]) * (1 if "large" in a[0] else 8)
                                                                                          for a, b in zip(alone, there)))


@pytest.mark.parametrize("shapes,pieces,others", [
    ("1536x1536,1530x1700", 252, None), ("1900x3000,1600x2000", 226, None), ("2600x2600,2600x2700", 242, None), ("40x70,2000x4200,12x2000,4200x40", 216, "1"),
    ("300x9000,2700x2600,2600x2600" + ",480x500" * 8, 242, "2"), ("100x130,1x1,333x777", 0, "1"), ("1000x1024,1000x1024,1000x1024", 0, "2")])
def test_symmetric_products_take_their_forms(launches, shapes, pieces, others):
    """The calls of test_gpu_memory_paths.py: workgroups of the pieces, tiles of the others in blocks."""
    found = launches("muon " + shapes)
    for product in ("(MuonProduct)0", "(MuonProduct)1"):
        assert {groups for kernel, arguments, groups in found if kernel == "muon_large_kernel" and arguments[0] == product} == ({pieces} if pieces else set())
        assert {arguments[1] for kernel, arguments, _ in found if kernel == "muon_product_kernel" and arguments[0] == product} == ({others} if others else set())


def _apply(found):
    """The kernels of the product with X, each once, with their tiles and workgroups."""
    return sorted({(kernel, arguments[1:2], groups) for kernel, arguments, groups in found if arguments[0] == "(MuonProduct)2"})


@pytest.mark.parametrize("large", ["2048x4096", "4096x2048", "2048x8192", "4096x4096"])
@pytest.mark.parametrize("small", ["30x100", "2048x12", "512x2048", "12x12,1x1", "300x200,200x300,12x300"])
def test_a_small_matrix_adds_no_round_to_a_large_ones_product(launches, large, small):
    """Tiles of 256 x 128 that are as many as the compute units, or twice as many: one more would take as long as all of them."""
    alone, beside = _apply(launches("muon " + large)), small.split(",")
    (kernel, _, groups), = alone
    assert kernel == "muon_large_kernel" and groups % 256 == 0
    for together in ([large] + beside, beside + [large], beside[:1] + [large] + beside[1:]):
        found = _apply(launches("muon " + ",".join(together)))
        assert [x for x in found if x[0] == kernel] == alone and any(x[0] == "muon_product_kernel" for x in found)


@pytest.mark.parametrize("shapes,groups,others", [
    ("3000x3000", None, "2"), ("2900x2900", None, "2"), ("2600x3400", None, "2"), ("4096x3000", 384, None), ("3200x3200", None, "2"), ("2600x4096", 352, None), ("3456x3456", 378, None), ("1500x3500", 168, None), ("3500x3500", 392, None), ("2048x3900", 248, None),
    ("2300x3000", 216, None), ("2048x2048", None, "2"), ("2047x4065", 256, None), (",".join(["500x520"] * 31 + ["40x33"]), None, "2"), ("2048x4096,1900x1900", 256, "2"),
    ("2048x4096,333x100", 256, "1"), ("777x333,235x512,333x1001,30x100", None, "1"), ("30x100,2040x4090,300x200", 256, "1"), ("2048x2000,1900x600,2000x2048", 256, "2")])
def test_products_with_x_take_their_forms(launches, shapes, groups, others):
    found = _apply(launches("muon " + shapes))
    assert [x[2] for x in found if x[0] == "muon_large_kernel"] == ([groups] if groups else [])
    assert [x[1] for x in found if x[0] == "muon_product_kernel"] == ([(others,)] if others else [])


@pytest.mark.parametrize("dtype,T,N,D,layout,forward,backward", [
    (BF16, 4096, 4, 1024, _side_by_side, 1024, ("8", "4", 32)), (F32, 2500, 6, 896, _side_by_side, None, ("8", "4", 20)), (F16, 3001, 5, 1280, _side_by_side, None, ("8", "4", 24)),
    (F32, 9000, 2, 64, _side_by_side, 282, ("4", "4", 141)), (BF16, 12345, 1, 40, _side_by_side, 193, ("4", "4", 193)), (F16, 20000, 3, 20, _by_sequence, 939, ("4", "4", 313))])
def test_long_sequences_take_their_pieces(launches, dtype, T, N, D, layout, forward, backward):
    """The calls of test_gpu_memory_paths.py: forward workgroups; backward steps of a lane, wavefronts, pieces of a sequence."""
    tiles = N * ((D + 63) // 64)
    found = launches(layout("forward", dtype, T, N, D))
    assert [kernel for kernel, _, _ in found] == ["recurrence_kernel", "recurrence_join_kernel", "recurrence_kernel"]
    assert forward is None or found[0][2] == found[2][2] == forward
    found = launches(layout("backward", dtype, T, N, D))
    assert [kernel for kernel, _, _ in found] == ["recurrence_backward_kernel", "recurrence_join_kernel", "recurrence_backward_kernel"]
    steps, waves, pieces = backward
    assert all(arguments[1:3] == (steps, waves) and groups == tiles * pieces for kernel, arguments, groups in found if kernel == "recurrence_backward_kernel")
