"""Operators of a model's layers, what can be checked without a GPU: refusals of the C entry points and of the binding,
sizes of workspaces, and the arithmetic by which ragged groups are cut into slices."""
import ctypes as C
import os

import numpy as np
import pytest

from paper_2211_00188_amd import engine as E
from paper_2211_00188_amd import layers as L

pytestmark = pytest.mark.skipif(not os.path.exists(E.LIB_PATH), reason="libadacgd.so not built")

P = 4096          # an address that is aligned and that no refused call reads
ARG, ALLOC = 1, 3


def T(data=P, dtype=0, stride=64, group_stride=0, pad=0):
    return C.byref(L.Tensor(data, dtype, pad, stride, group_stride))


def refused(name, args, code=ARG, text=""):
    lib = L._library()
    assert getattr(lib, name)(*args) == code, lib.adacgd_last_error(None)
    message = lib.adacgd_last_error(None).decode()
    assert text in message and message, message


def test_every_entry_point_is_bound():
    assert set(L.ARGTYPES) <= set(E.EXPORTS)


GOOD = dict(product=0, rows=10, groups=2, n=64, k=32, offsets=P, a=T(), b=T(group_stride=4096), c=T(), ws=None, size=0, stream=None)


@pytest.mark.parametrize("bad,code,text", [
    (dict(product=3), ARG, "product"), (dict(product=-1), ARG, "product"), (dict(rows=-1), ARG, "rows"), (dict(rows=1 << 31), ARG, "rows"),
    (dict(groups=0), ARG, "groups"), (dict(groups=1 << 31), ARG, "groups"), (dict(n=0), ARG, "n must"), (dict(k=0), ARG, "k must"),
    (dict(n=(1 << 24) + 1), ARG, "n must"), (dict(offsets=None), ARG, "offsets"), (dict(a=None), ARG, "a is null"),
    (dict(a=T(data=None)), ARG, "a: data"), (dict(a=T(dtype=3)), ARG, "type"), (dict(a=T(dtype=-1)), ARG, "type"), (dict(a=T(pad=1)), ARG, "pad"),
    (dict(a=T(data=P + 2)), ARG, "aligned"), (dict(a=T(stride=31)), ARG, "stride"), (dict(a=T(stride=1 << 31)), ARG, "stride"),
    (dict(b=T(group_stride=-64)), ARG, "group_stride"), (dict(b=T(dtype=1)), ARG, "differ in type"), (dict(c=T(dtype=1)), ARG, "c has neither"),
    (dict(c=T(stride=63)), ARG, "stride"),
    (dict(product=2, c=T(stride=64, group_stride=63 * 64)), ARG, "smaller than a matrix"), (dict(product=2, c=T(group_stride=0)), ARG, "smaller"),
])
def test_bad_products_are_refused(bad, code, text):
    refused("adacgd_group_matmul", list(dict(GOOD, **bad).values()), code, text)


def test_products_without_rows_need_no_data():
    lib = L._library()
    for product in (0, 1):
        args = dict(GOOD, product=product, rows=0, a=T(data=None), c=T(data=None))
        assert lib.adacgd_group_matmul(*args.values()) == 0, lib.adacgd_last_error(None)


def test_workspace_of_the_products():
    lib, n = L._library(), C.c_int64(-1)
    for product in (0, 1):
        assert lib.adacgd_group_matmul_workspace_bytes(product, 1, 100000, 7, 512, 512, C.byref(n)) == 0 and n.value == 0
    assert lib.adacgd_group_matmul_workspace_bytes(2, 1, 100000, 7, 512, 512, C.byref(n)) == 0 and n.value >= 0 and n.value % 256 == 0
    refused("adacgd_group_matmul_workspace_bytes", [0, 0, 1, 1, 1, 1, None], ARG, "bytes")
    refused("adacgd_group_matmul_workspace_bytes", [0, 5, 1, 1, 1, 1, C.byref(n)], ARG, "type")
    refused("adacgd_group_matmul_workspace_bytes", [4, 0, 1, 1, 1, 1, C.byref(n)], ARG, "product")


NORM = dict(rows=10, d=64, x=T(), weight=None, bias=None, eps=1e-5, y=T(), mean=None, rstd=None, stream=None)


@pytest.mark.parametrize("bad,text", [
    (dict(rows=-1), "rows"), (dict(d=0), "d must"), (dict(d=1 << 25), "d must"), (dict(x=None), "x is null"), (dict(y=T(dtype=1)), "differ in type"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"), (dict(mean=P), "together"), (dict(rstd=P), "together"),
    (dict(x=T(stride=10)), "stride"), (dict(y=T(data=P + 1)), "aligned"),
])
def test_bad_norms_are_refused(bad, text):
    refused("adacgd_layer_norm", list(dict(NORM, **bad).values()), ARG, text)


BACK = dict(rows=10, groups=2, d=64, offsets=P, dy=T(), x=T(), weight=None, mean=P, rstd=P, dx=T(), dw=T(), db=T(), ws=None, size=0, stream=None)


@pytest.mark.parametrize("bad,text", [
    (dict(groups=0), "groups"), (dict(offsets=None), "offsets"), (dict(dy=T(dtype=1)), "differ in type"), (dict(dx=T(dtype=2)), "differ in type"),
    (dict(mean=None), "mean or rstd"), (dict(rstd=None), "mean or rstd"), (dict(dw=T(dtype=1)), "fp32"), (dict(db=T(stride=63)), "dbias: stride"),
    (dict(dw=T(data=None)), "dweight: data"),
])
def test_bad_norm_gradients_are_refused(bad, text):
    refused("adacgd_layer_norm_backward", list(dict(BACK, **bad).values()), ARG, text)


DROP = dict(rows=10, d=64, x=T(), residual=None, out=T(), p=0.5, seed=1, step=0, step_dev=None, layer=0, first=0, stream=None)


@pytest.mark.parametrize("bad,text", [
    (dict(p=-0.01), "p must"), (dict(p=1.01), "p must"), (dict(p=float("nan")), "p must"), (dict(layer=0xFFFFFFFF), "layer"),
    (dict(residual=T(dtype=1)), "differ in type"), (dict(out=T(dtype=1)), "differ in type"), (dict(out=None), "out is null"),
    (dict(residual=T(stride=3)), "residual: stride"),
])
def test_bad_dropout_is_refused(bad, text):
    refused("adacgd_dropout", list(dict(DROP, **bad).values()), ARG, text)


LOSS = dict(tokens=10, pairs=2, v=64, logits=T(), targets=P, offsets=P, ref=None, beta=0.1, smoothing=0.0, loss=P, margin=P, logp=P, lse=P,
            ws=P, size=1 << 40, stream=None)
GRAD = dict(tokens=10, pairs=2, v=64, dloss=P, logits=T(), targets=P, offsets=P, margin=P, lse=P, beta=0.1, smoothing=0.0, out=T(), stream=None)
SHARED = [(dict(tokens=-1), "tokens"), (dict(pairs=-1), "pairs"), (dict(v=0), "v must"), (dict(targets=None), "targets"), (dict(offsets=None), "offsets"),
          (dict(beta=float("nan")), "beta"), (dict(beta=float("inf")), "beta"), (dict(smoothing=-0.1), "smoothing"), (dict(smoothing=1.5), "smoothing"),
          (dict(smoothing=float("nan")), "smoothing"), (dict(logits=T(stride=8)), "stride")]


@pytest.mark.parametrize("bad,text", SHARED + [(dict(loss=None), "loss"), (dict(margin=None), "margin"), (dict(logp=None), "logp"), (dict(lse=None), "lse")])
def test_bad_preference_losses_are_refused(bad, text):
    refused("adacgd_preference_loss", list(dict(LOSS, **bad).values()), ARG, text)


@pytest.mark.parametrize("bad,text", SHARED + [(dict(dloss=None), "dloss"), (dict(margin=None), "margin"), (dict(lse=None), "lse"),
                                               (dict(out=T(dtype=1)), "differ in type")])
def test_bad_preference_gradients_are_refused(bad, text):
    refused("adacgd_preference_loss_backward", list(dict(GRAD, **bad).values()), ARG, text)


def test_the_binding_refuses_host_tensors():
    import torch
    x, off = torch.zeros(4, 8), torch.tensor([0, 4])
    for call in (lambda: L.group_matmul(x, x[None], off), lambda: L.group_matmul_dw(x, x, off), lambda: L.layer_norm(x),
                 lambda: L.dropout(x, 0.5, 1), lambda: L.preference_loss(x, off, off)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()


@pytest.mark.parametrize("shift", [4, 5, 6, 7, 8, 13])
def test_numbers_of_slices_ascend_without_a_prefix_sum(shift):
    """(offset >> shift) + group + j: ascending, one at least for every group, below (rows >> shift) + groups."""
    rng = np.random.default_rng(shift)
    for trial in range(200):
        groups = int(rng.integers(1, 40))
        sizes = rng.integers(0, 4 << shift, groups) * (rng.random(groups) < 0.8)
        first = int(rng.integers(0, 3 << shift))
        o = np.concatenate([[first], first + np.cumsum(sizes)])
        rows = int(o[-1] + rng.integers(0, 2 << shift))
        numbers = [(int(o[g]) >> shift) + g + j for g in range(groups) for j in range(max(1, -(-int(sizes[g]) >> shift)))]
        assert all(a < b for a, b in zip(numbers, numbers[1:])) and numbers[-1] < (rows >> shift) + groups


@pytest.mark.parametrize("shift", [8, 9, 11, 13])
def test_places_of_cut_groups_sums_do_not_meet(shift):
    """2 (first row >> shift) + j for the slices of groups of more than 2^shift rows: no two alike, all below 2 (rows >> shift) + 1."""
    rng = np.random.default_rng(shift)
    for trial in range(300):
        groups = int(rng.integers(1, 30))
        sizes = (rng.integers(0, 4 << shift, groups) * (rng.random(groups) < 0.7)).astype(int)
        sizes[rng.random(groups) < 0.3] = (1 << shift) + int(rng.integers(-1, 2))
        o = int(rng.integers(0, 2 << shift)) + np.concatenate([[0], np.cumsum(sizes)])
        rows = int(o[-1])
        places = [2 * (int(o[g]) >> shift) + j for g in range(groups) if sizes[g] > 1 << shift for j in range(-(-int(sizes[g]) >> shift))]
        assert len(set(places)) == len(places) and max(places, default=0) < 2 * (rows >> shift) + 1


def test_the_preference_workloads_parts_are_views_in_order():
    from paper_2211_00188_amd import workloads as W
    wl = W.preference(n=3, pairs=7, width=8, vocab=11, length=6)
    assert wl.d == 8 + 8 + 64 + 88 == wl.x0.size and wl.worker_pairs[-1] == 7 and (np.diff(wl.worker_pairs) > 0).all()
    ext = np.zeros((3, wl.d), np.float32)
    for k, part in enumerate(wl.parts(ext).values()):
        part[...] = k + 1                                       # written into the array itself
    assert ext.tolist() == [[1.0] * 8 + [2.0] * 8 + [3.0] * 64 + [4.0] * 88] * 3
    assert wl.worker_rows()[-1] == len(wl.targets) == len(wl.features) == len(wl.ref) and wl.worker_rows()[0] == 0
    again = W.preference(n=3, pairs=7, width=8, vocab=11, length=6)
    assert np.array_equal(again.features, wl.features) and np.array_equal(again.targets, wl.targets)


@pytest.fixture(scope="module")
def helpers(tmp_path_factory):
    """The host side of csrc/layers.h's numbering of slices, as it is compiled."""
    import shutil
    import subprocess
    from paper_2211_00188_amd import build as B
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not shutil.which(hipcc):
        pytest.skip("no hipcc")
    where = tmp_path_factory.mktemp("helpers")
    names = {"slice_numbers": 3, "first_number": 3, "part_number": 2, "part_numbers": 2}
    with open(where / "helpers.hip", "w") as f:
        f.write('#include "%s/layers.h"\n' % B.CSRC)
        for name, count in names.items():
            longs = ["int64_t a", "int64_t b"][:count - 1]
            f.write('extern "C" int64_t t_%s(%s, int shift) { return adacgd::%s(%s, shift); }\n'
                    % (name, ", ".join(longs), name, ", ".join(v[-1] for v in longs)))
    subprocess.run([hipcc, "--cuda-host-only", "-std=c++17", "-fPIC", "-shared", "-o", str(where / "helpers.so"), str(where / "helpers.hip")],
                   check=True, capture_output=True)
    lib = C.CDLL(str(where / "helpers.so"))
    for name, count in names.items():
        f = getattr(lib, "t_" + name)
        f.argtypes, f.restype = [C.c_int64] * (count - 1) + [C.c_int], C.c_int64
    return lib


@pytest.mark.parametrize("shift", [2, 4, 6, 7, 8, 13])
def test_the_librarys_numbers_of_slices_are_within_its_launches_and_workspaces(helpers, shift):
    """Every slice of every group has a number of its own below what is launched, and every slice of a cut group a place of its own
    inside the workspace, to the last row."""
    rng = np.random.default_rng(100 + shift)
    for trial in range(300):
        groups = int(rng.integers(1, 40))
        sizes = (rng.integers(0, 5 << shift, groups) * (rng.random(groups) < 0.75)).astype(int)
        sizes[rng.random(groups) < 0.2] = (1 << shift) + int(rng.integers(-1, 2))
        o = int(rng.integers(0, 3 << shift)) + np.concatenate([[0], np.cumsum(sizes)])
        rows = int(o[-1]) + int(rng.integers(0, 3)) * int(rng.integers(0, 2 << shift))
        count = [max(1, -(-int(m) >> shift)) for m in sizes]
        numbers = [helpers.t_first_number(int(o[g]), g, shift) + j for g in range(groups) for j in range(count[g])]
        assert numbers[0] >= 0 and all(a < b for a, b in zip(numbers, numbers[1:])) and numbers[-1] < helpers.t_slice_numbers(rows, groups, shift)
        places = [helpers.t_part_number(int(o[g]), shift) + j for g in range(groups) if sizes[g] > 1 << shift for j in range(count[g])]
        assert len(set(places)) == len(places) and max(places, default=0) < helpers.t_part_numbers(rows, shift) and min(places, default=0) >= 0


@pytest.mark.parametrize("sizes,n,k", [([65536], 512, 512), ([262144], 64, 64), ([30000] + [2] * 300, 256, 256), ([16384], 1032, 1040)])
def test_workspace_of_cut_groups_holds_two_slices_of_the_longest(sizes, n, k):
    """A group that is cut has two slices at least, and their partial sums are fp32 matrices side by side."""
    lib, size = L._library(), C.c_int64(-1)
    for dtype in (0, 1, 2):
        assert lib.adacgd_group_matmul_workspace_bytes(2, dtype, sum(sizes), len(sizes), n, k, C.byref(size)) == 0
        assert size.value >= 2 * n * k * 4 and size.value % 256 == 0
    assert lib.adacgd_layer_norm_backward_workspace_bytes(sum(sizes), len(sizes), n, C.byref(size)) == 0
    assert size.value >= 2 * 2 * n * 4


@pytest.mark.parametrize("eps", [1e-46, 5e-324, 1e39])
def test_norms_refuse_an_eps_that_fp32_has_no_number_for(eps):
    refused("adacgd_layer_norm", list(dict(NORM, eps=eps).values()), ARG, "eps")
