"""MXFP4 rows, the product with them and the quantised cache without a GPU: sizes, refusals, and the plain forms."""
import numpy as np
import pytest
import torch

from paper_2508_05700_amd import binding as b
from tests import mx_plain

OK, INVALID, UNSUPPORTED = 0, -1, -2
FAKE = 0x1000   # a non-null, aligned address; every call that uses it has an invalid argument or nothing to do
F32, BF16, INT8, INT4, INT4R64, MX = 0, 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def L():
    return b.lib()


def test_row_bytes(L):
    assert [L.emb_row_bytes(D, MX) for D in (32, 64, 96, 128, 256, 512, 1024, 4096)] == [32, 48, 64, 80, 144, 272, 544, 2176]
    assert L.emb_row_bytes(16, MX) == 0 and L.emb_row_bytes(33, MX) == 0 and L.emb_row_bytes(0, MX) == 0
    assert L.emb_row_bytes(64, 5) == 0 and L.emb_row_bytes(64, 7) == 0
    assert all(L.emb_row_bytes(D, MX) == mx_plain.row_bytes(D) for D in range(32, 2049, 32))


def test_quantize_refusals(L):
    q = L.emb_quantize_rows
    assert q(FAKE, 10, 48, MX, FAKE, None) == UNSUPPORTED and q(FAKE, 10, 65568, MX, FAKE, None) == UNSUPPORTED
    assert q(FAKE, 10, 0, MX, FAKE, None) == INVALID and q(FAKE, 0, 2048, MX, FAKE, None) == OK
    f = L.emb_quantize_rows_from
    args = lambda **k: [k.get("src", FAKE), k.get("sd", F32), k.get("stride", 64), k.get("n", 4), k.get("D", 64), k.get("dt", MX),
                        k.get("dst", FAKE), None]
    assert f(*args(n=0)) == OK
    assert f(*args(n=-1)) == INVALID and f(*args(src=None)) == INVALID and f(*args(dst=None)) == INVALID
    assert f(*args(sd=MX)) == INVALID and f(*args(sd=INT8)) == INVALID and f(*args(sd=9)) == INVALID
    assert f(*args(dt=F32)) == INVALID and f(*args(dt=5)) == INVALID
    assert f(*args(stride=63)) == INVALID and f(*args(stride=66)) == INVALID      # shorter than a row; not whole 16 bytes
    assert f(*args(sd=BF16, stride=68)) == INVALID and f(*args(stride=1 << 62)) == INVALID
    assert f(*args(src=FAKE + 8)) == INVALID and f(*args(dst=FAKE + 4)) == INVALID
    assert f(*args(n=1 << 31)) == UNSUPPORTED and f(*args(D=40, stride=40)) == UNSUPPORTED
    assert f(*args(D=1040, stride=1040, dt=INT8)) == UNSUPPORTED
    d = L.emb_dequantize_rows
    args = lambda **k: [k.get("src", FAKE), k.get("dt", MX), k.get("n", 4), k.get("D", 64), k.get("dst", FAKE), k.get("dd", F32),
                        k.get("stride", 64), None]
    assert d(*args(n=0)) == OK
    assert d(*args(n=-1)) == INVALID and d(*args(src=None)) == INVALID and d(*args(dst=None)) == INVALID
    assert d(*args(dt=F32)) == INVALID and d(*args(dd=MX)) == INVALID and d(*args(dd=INT4)) == INVALID
    assert d(*args(stride=60)) == INVALID and d(*args(dd=BF16, stride=68)) == INVALID and d(*args(dst=FAKE + 4)) == INVALID
    assert d(*args(D=48, stride=48)) == UNSUPPORTED and d(*args(n=1 << 31)) == UNSUPPORTED


def test_lookups_take_the_type_up_to_1024_elements(L):
    d = np.zeros(1, dtype=b.TABLE_DESC)
    d["num_rows"], d["weights"] = 10, FAKE
    assert L.emb_tables_init(d.ctypes.data, 1) == OK
    f = L.emb_bag_forward
    go = lambda D, B=4: f(d.ctypes.data, FAKE, 1, D, MX, FAKE, FAKE, B, 8, 0, FAKE if B == 0 else None, None, None)
    assert go(48) == UNSUPPORTED and go(1056) == UNSUPPORTED and go(1024) == INVALID and go(96, 0) == OK
    assert L.emb_bag_backward_workspace_bytes(1, 4, 8, 10, 64, MX) == 0          # not trained
    assert L.emb_cache_build(FAKE, 100, 48, MX, FAKE, 10, FAKE, FAKE, None, None) == UNSUPPORTED


def test_product_refusals(L):
    f = L.emb_rows_product
    args = lambda **k: [k.get("x", FAKE), k.get("xd", F32), k.get("xs", 64), k.get("M", 4), k.get("w", FAKE), k.get("N", 8),
                        k.get("D", 64), k.get("out", FAKE), k.get("od", F32), k.get("os", 8), None]
    assert f(*args(M=0)) == OK and f(*args(N=0, os=0)) == OK
    assert f(*args(M=-1)) == INVALID and f(*args(N=-1)) == INVALID
    assert f(*args(x=None)) == INVALID and f(*args(w=None)) == INVALID and f(*args(out=None)) == INVALID
    assert f(*args(xd=INT8)) == INVALID and f(*args(xd=5)) == INVALID and f(*args(od=MX)) == INVALID
    assert f(*args(xs=32)) == INVALID and f(*args(xs=66)) == INVALID and f(*args(xd=BF16, xs=68)) == INVALID
    assert f(*args(os=7)) == INVALID
    assert f(*args(x=FAKE + 8)) == INVALID and f(*args(w=FAKE + 8)) == INVALID and f(*args(out=FAKE + 2)) == INVALID
    assert f(*args(out=FAKE + 1, od=BF16)) == INVALID
    assert f(*args(D=48, xs=48)) == UNSUPPORTED and f(*args(D=65568, xs=65568)) == UNSUPPORTED and f(*args(D=0)) == INVALID
    assert f(*args(M=1 << 31)) == UNSUPPORTED and f(*args(N=1 << 31, os=1 << 31)) == UNSUPPORTED
    assert f(*args(D=32, M=1, N=(1 << 31) - 1, os=1 << 31)) == UNSUPPORTED       # more threads than a grid holds
    assert f(*args(xd=MX, xs=0, M=0)) == OK                                      # the stride of MXFP4 rows is their size


def test_quantized_cache_refusals(L):
    f = L.emb_cache_build_quantized
    args = lambda **k: [k.get("table", FAKE), k.get("R", 100), k.get("D", 64), k.get("dt", F32), k.get("cd", MX),
                        k.get("hot", FAKE), k.get("n", 10), k.get("rows", FAKE), k.get("index", FAKE), None, None]
    assert f(*args(dt=INT8)) == INVALID and f(*args(cd=F32)) == INVALID and f(*args(cd=BF16)) == INVALID and f(*args(cd=5)) == INVALID
    assert f(*args(D=48)) == UNSUPPORTED and f(*args(D=40, cd=INT8)) == UNSUPPORTED and f(*args(D=1056)) == UNSUPPORTED
    assert f(*args(n=101)) == INVALID and f(*args(n=-1)) == INVALID and f(*args(R=0)) == INVALID
    assert f(*args(table=None)) == INVALID and f(*args(hot=None)) == INVALID and f(*args(rows=None)) == INVALID
    assert f(*args(index=None)) == INVALID and f(*args(table=FAKE + 4)) == INVALID
    g = L.emb_cache_rebuild_quantized
    args = lambda **k: [FAKE, 100, 64, k.get("dt", F32), k.get("cd", MX), k.get("orows", 0x2000), k.get("oindex", 0x3000),
                        k.get("on", 10), FAKE, 10, FAKE, FAKE, None, None, None]
    assert g(*args(oindex=None)) == INVALID and g(*args(orows=None)) == INVALID and g(*args(on=101)) == INVALID
    assert g(*args(orows=FAKE)) == INVALID and g(*args(oindex=FAKE)) == INVALID      # the older cache is read meanwhile
    assert g(*args(cd=F32)) == INVALID
    h = L.emb_bag_forward_cached_quantized
    args = lambda **k: [k.get("table", FAKE), k.get("R", 100), k.get("D", 64), k.get("dt", F32), k.get("cd", MX), k.get("rows", FAKE),
                        k.get("index", FAKE), k.get("n", 10), k.get("ids", FAKE), k.get("off", FAKE), k.get("B", 4), k.get("nnz", 8),
                        k.get("mode", 0), k.get("out", FAKE), None, None, None]
    assert h(*args(B=0)) == OK
    for bad in (dict(dt=MX), dict(cd=F32), dict(table=None), dict(index=None), dict(rows=None), dict(ids=None), dict(off=None),
                dict(out=None), dict(out=FAKE + 4), dict(mode=2), dict(mode=0x100), dict(B=-1), dict(nnz=-1), dict(R=0), dict(n=-1)):
        assert h(*args(**bad)) == INVALID, bad
    assert h(*args(D=48)) == UNSUPPORTED
    hh = L.emb_bag_forward_cached_quantized_hashed
    a = args(ids=None)
    assert hh(*(a[:8] + [7] + a[8:])) == INVALID


def test_a_quantized_cache_that_does_not_fit_its_tensors_is_refused():
    # 100 rows of 64 elements: rows of 48 bytes, an index of 2 entries of 16
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8)
    ids, offs, out = torch.zeros(8, dtype=torch.int64), torch.zeros(5, dtype=torch.int64), torch.zeros(4, 64)
    lookup = lambda rows, index: b.emb_bag_forward_cached_quantized(4096, 100, 64, "f32", "mxfp4", rows, index, 10, ids, offs, 4,
                                                                      "sum", out)
    hashed = lambda rows, index: b.emb_bag_forward_cached_quantized_hashed(4096, 100, 64, "f32", "mxfp4", rows, index, 10, 7, ids,
                                                                             offs, 4, "sum", out)
    build = lambda rows, index: b.emb_cache_build_quantized(4096, 100, 64, "f32", "mxfp4", ids, rows, index)
    rebuild = lambda rows, index: b.emb_cache_rebuild_quantized(4096, 100, 64, "f32", "mxfp4", rows, index, 10, ids, u8(480), u8(32))
    rebuild_to = lambda rows, index: b.emb_cache_rebuild_quantized(4096, 100, 64, "f32", "mxfp4", u8(480), u8(32), 10, ids, rows, index)
    for call, need in ((lookup, 480), (hashed, 480), (build, 8 * 48), (rebuild, 480), (rebuild_to, 8 * 48)):
        with pytest.raises(TypeError, match="rows too small"):
            call(u8(need - 1), u8(32))
        with pytest.raises(TypeError, match="index too small"):
            call(u8(need), u8(31))


def test_plain_form_of_the_definition():
    # ties, saturation, the scale of a block, and that values read back are fixed points
    x = np.zeros((2, 32))
    x[0, :14] = [6, 7.99, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -0.75, -5, 0.26, -0.0]
    codes, scales = mx_plain.quantize(x)
    assert scales.tolist() == [[127], [0]]
    assert mx_plain.GRID[codes[0, :14] & 7].tolist() == [6, 6, 4, 4, 2, 2, 1, 1, 0, 0, 1, 4, 0.5, 0] and codes[0, 13] == 8
    rng = np.random.default_rng(1)
    y = rng.standard_normal((20, 64)) * 2.0 ** rng.integers(-100, 100, (20, 1))
    rows = mx_plain.pack(*mx_plain.quantize(y))
    v = mx_plain.values(rows, 64)
    step = np.repeat(2.0 ** (rows[:, 32:34].astype(float) - 127), 32, axis=1)
    assert np.all(np.abs(v - y) <= np.where(np.abs(y) > 6 * step, 2, 1) * step)      # half a step of 2 at most, 2 where it saturates
    assert np.array_equal(mx_plain.values(mx_plain.pack(*mx_plain.quantize(v)), 64), v)
