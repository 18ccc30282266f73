"""MXFP4 rows at the edges of their range, of the kernels' rules by size and of a launch, against the definition in 64 bits.

Tolerances are those of tests/test_mx_rows.py where sums are random; where a sum has one element it is exact and compared
as such."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2508_05700_amd import binding as emb  # noqa: E402
from tests import harness as H  # noqa: E402
from tests import mx_plain as mx  # noqa: E402

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}

# Sizes of the product with an fp32 or bf16 x, by the kernel that takes the one or the other: rows straight from memory, one
# wavefront or several a tile; x in LDS, whole and in parts of K; half tiles; whole tiles.
PRODUCTS = [(3, 40, 96), (20, 70, 64), (5, 64, 1056), (160, 1024, 544), (20, 6000, 512), (16, 33_000, 4128), (40, 17_000, 1024),
            (50, 20_700, 288), (50, 66_000, 544), (129, 10_400, 288), (260, 33_000, 544), (300, 20_600, 96)]


def _infinite(rows, D):
    """Values of packed rows as fp32 has them: what lies beyond its range is infinite."""
    v = mx.values(rows, D)
    return np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,D", PRODUCTS)
def test_product_with_rows_beyond_the_range_of_fp32(M, N, D, kind, out):
    # scale bytes 253 and 254 with codes up to 6: infinite elements, which meet x of few bits (its lower parts are zero), of all
    # bits, and zeros; finite ones beside them; rows that have none keep what they have without such neighbours
    rng = np.random.default_rng(M + N + D)
    w = mx.random_rows(rng, N, D, 100, 110)
    plain = w.copy()
    far = np.unique(np.concatenate((rng.integers(0, N, 6), [0, N - 1])))
    for i, n in enumerate(far):
        b = int(rng.integers(0, D // 32))
        w[n, D // 2 + b] = 253 + i % 2
        if i % 3:
            w[n, 16 * b:16 * b + 16] &= 0x99            # codes 0 and 1: large, and finite
        if i % 3 == 1:                                  # and one that is infinite
            w[n, 16 * b + int(rng.integers(0, 16))] |= rng.choice(np.array([6, 7, 0x60, 0x70], dtype=np.uint8))
    x = rng.integers(1, 128, (M, D)).astype(np.float32) * np.float32(2.0 ** -20) * rng.choice([-1, 1], (M, D)).astype(np.float32)
    x[M // 2] *= np.float32(1.0 + 2.0 ** -23)           # (bf16: as it was)
    x[M - 1] = 0.0
    x = torch.from_numpy(x).to(TORCH[kind])
    got, base = (torch.full((M, N), 3.0, dtype=TORCH[out], device=H.DEV) for _ in range(2))
    emb.emb_rows_product(x.to(H.DEV), H.dev(w), D, got)
    emb.emb_rows_product(x.to(H.DEV), H.dev(plain), D, base)
    got, base = got.cpu(), base.cpu()
    rest = np.setdiff1d(np.arange(N), far)
    assert torch.equal(got[:, rest], base[:, rest])
    xv, g = x.double().numpy(), got.double().numpy()
    for n in far:
        v = _infinite(w[n:n + 1], D)[0]
        with np.errstate(invalid="ignore"):
            ref = (xv * v).sum(1)
        assert np.array_equal(np.isnan(ref), np.isnan(g[:, n])), n
        inf = np.isinf(ref)
        assert np.array_equal(ref[inf], g[inf, n]), n
        keep = np.isfinite(ref)
        # one addition an element (three for fp32) of at most one step of the sum of magnitudes; then bf16's half step
        tol = D * (3 if kind == "f32" else 1) * 2.0 ** -23 * (np.abs(xv[keep]) @ np.where(np.isinf(v), 0, np.abs(v)))
        if out == "bf16":
            tol = tol + 2.0 ** -8 * (np.abs(ref[keep]) + tol)
        assert np.all(np.abs(g[keep, n] - ref[keep]) <= tol), n


@pytest.mark.parametrize("M,N,D", PRODUCTS)
def test_product_of_fp32_keeps_every_bit_in_every_kernel(M, N, D):
    # one element of 24 bits a row of x, by a power of two: the product is exact, and each of the three parts of x takes part in
    # it.  Over the passes the element goes over every place of a block, over the blocks and over the rows of a tile.
    rng = np.random.default_rng(M * 3 + N + D)
    w = mx.pack(rng.choice(np.array([1, 2, 4, 6, 9, 10, 12, 14], dtype=np.uint8), (N, D)), rng.integers(120, 130, (N, D // 32), dtype=np.uint8))
    wv = torch.from_numpy(mx.values(w, D)).to(H.DEV)
    wd = H.dev(w)
    rows = torch.arange(M, device=H.DEV)
    got = torch.empty((M, N), device=H.DEV)
    for k in range(8):
        at = torch.from_numpy((np.arange(M) * 37 + k * (D // 8 + 5) + rng.integers(0, D)) % D).to(H.DEV)
        bits = rng.integers(1 << 23, 1 << 24, M) | 0x10101          # a bit at the lower end of every part
        v = torch.from_numpy(bits * 2.0 ** rng.integers(-40, 10, M).astype(float) * rng.choice([-1, 1], M)).to(H.DEV)
        x = torch.zeros((M, D), device=H.DEV)
        x[rows, at] = v.float()
        emb.emb_rows_product(x, wd, D, got)
        assert torch.equal(got.double(), v[:, None] * wv[:, at].t()), k


@pytest.mark.parametrize("kind,M,N", [("f32", 70, 20_600), ("f32", 49, 20_600), ("bf16", 70, 300), ("bf16", 33, 130)])
def test_product_of_many_rows_very_far_apart(kind, M, N):
    # more rows of x than the sizes alone would send to the kernel that takes rows more than 4 MB apart
    D, stride = 64, 3 << 20
    rng = np.random.default_rng(M + N)
    far = torch.full((M, stride), float("nan"), dtype=TORCH[kind], device=H.DEV)
    x = torch.from_numpy(rng.standard_normal((M, D)).astype(np.float32)).to(TORCH[kind])
    far[:, :D] = x.to(H.DEV)
    w = mx.random_rows(rng, N, D, 118, 129)
    o = torch.empty((M, N), device=H.DEV)
    emb.emb_rows_product(far[:, :D], H.dev(w), D, o)
    xv, wv = x.double().numpy(), mx.values(w, D)
    tol = D * (3 if kind == "f32" else 1) * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T)
    assert np.all(np.abs(o.cpu().double().numpy() - xv @ wv.T) <= tol)


@pytest.mark.parametrize("mode", ["sum", "mean"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q,D", [("int8", 16), ("int4", 16), ("int4r64", 16), ("int8", 48), ("int4", 80), ("mxfp4", 160), ("int8", 240),
                                 ("mxfp4", 256), ("int4", 272), ("mxfp4", 320), ("int4r64", 496), ("mxfp4", 544), ("int8", 1008)])
def test_quantized_cache_of_every_width(q, D, dtype, mode):
    # every number of lanes to a bag, filled and partly filled, bags from none to several batches of lookups
    rng = np.random.default_rng(D)
    R, B = 150, 41
    t = torch.from_numpy((rng.standard_normal((R, D)) * 2.0 ** rng.integers(-20, 20, (R, 1))).astype(np.float32)).to(TORCH[dtype]).to(H.DEV)
    lengths = rng.integers(0, 70, B)
    lengths[[0, 7, B - 1]] = 0, 0, 130
    off = np.concatenate(([0], np.cumsum(lengths))).astype(np.int64)
    raw = rng.integers(0, 1 << 63, size=int(off[-1]), dtype=np.int64)
    rows = torch.empty(raw.size, dtype=torch.int64, device=H.DEV)
    emb.emb_hash_ids(H.dev(raw), 5, R, rows)
    hot = np.sort(rng.choice(R, size=90, replace=False)).astype(np.int64)
    status = torch.zeros(1, dtype=torch.int32, device=H.DEV)
    hm = torch.zeros(2, dtype=torch.int64, device=H.DEV)
    cache = torch.empty((hot.size, emb.emb_row_bytes(D, q)), dtype=torch.uint8, device=H.DEV)
    index = torch.empty(emb.emb_cache_index_bytes(R), dtype=torch.uint8, device=H.DEV)
    emb.emb_cache_build_quantized(t.data_ptr(), R, D, dtype, q, H.dev(hot), cache, index, status)
    vals = t.double().cpu().numpy()
    packed = cache.cpu().numpy()
    vals[hot] = mx.values(packed, D) if q == "mxfp4" else mx.int_values(packed, D, q)
    r = rows.cpu().numpy()
    ref, mag = mx.pool(vals[r], off, mode)
    n = lengths[:, None]
    hits = int(np.isin(r, hot).sum())
    for call, ids in ((emb.emb_bag_forward_cached_quantized, (rows,)), (emb.emb_bag_forward_cached_quantized_hashed, (5, H.dev(raw)))):
        out = torch.full((1, B, D), 9.0, device=H.DEV)
        hm.zero_()
        call(t.data_ptr(), R, D, dtype, q, cache, index, hot.size, *ids, H.dev(off), B, mode, out, hm, status)
        got = out.cpu().numpy()[0]
        # a sum's additions and a mean's division, and of INT rows the fused multiply-add, of half a step each
        assert np.all(np.abs(got - ref) <= (n + 2) * 2.0 ** -24 * mag)
        assert (got[lengths == 0] == 0).all()
        assert hm.cpu().tolist() == [hits, r.size - hits]
    assert status.item() == 0


def test_product_of_more_threads_than_a_grid_holds():
    # 33 rows of fp32 x are three tiles by 128 rows of W: beyond 7.1e8 rows of W more than 2^32 threads
    M, N, D = 33, 730_000_000, 32
    rng = np.random.default_rng(9)
    at = np.unique(np.concatenate((rng.integers(0, N, 300), np.arange(N // 2 - 3000, N // 2 + 3000), [0, N - 1])))
    w = mx.random_rows(rng, at.size, D, 118, 129)
    w[:, 0] |= 0x11                                          # (no row of zeros)
    wd = torch.zeros((N, emb.emb_row_bytes(D, "mxfp4")), dtype=torch.uint8, device=H.DEV)
    where = torch.from_numpy(at).to(H.DEV)
    wd[where] = H.dev(w)
    x = torch.from_numpy(rng.standard_normal((M, D)).astype(np.float32))
    o = torch.full((M, N), 3.0, dtype=torch.bfloat16, device=H.DEV)
    emb.emb_rows_product(x.to(H.DEV), wd, D, o)
    xv, wv = x.double().numpy(), mx.values(w, D)
    got = o[:, where].cpu().double().numpy()
    ref, mag = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    tol = 3 * D * 2.0 ** -23 * mag
    assert np.all(np.abs(got - ref) <= tol + 2.0 ** -8 * (np.abs(ref) + tol))
    for m in range(M):                                       # every other row of W is zeros
        assert int(torch.count_nonzero(o[m])) == int(np.count_nonzero(got[m])), m


def test_int_rows_of_more_threads_than_a_grid_holds():
    # 64 threads a row of 528 elements: beyond 6.7e7 rows more than 2^32
    R, D, k, q = 68_000_000, 528, 300, "int4"
    rng = np.random.default_rng(10)
    at = np.unique(np.concatenate((rng.integers(0, R, k), np.arange((1 << 25) - k, (1 << 25) + k), np.arange((1 << 26) - k, (1 << 26) + k),
                                   np.arange(R - k, R))))
    where = torch.from_numpy(at).to(H.DEV)
    t = torch.from_numpy(rng.standard_normal((at.size, D)).astype(np.float32)).to(torch.bfloat16).to(H.DEV)
    src = torch.ones((R, D), dtype=torch.bfloat16, device=H.DEV)
    src[where] = t
    rows = torch.zeros((R, emb.emb_row_bytes(D, q)), dtype=torch.uint8, device=H.DEV)
    emb.emb_quantize_rows_from(src, q, rows)
    want = torch.empty((at.size, rows.shape[1]), dtype=torch.uint8, device=H.DEV)
    emb.emb_quantize_rows_from(t, q, want)
    assert torch.equal(rows[where], want)
    # (every other row is constant: scale and bias 1, codes 0)
    header = rows[:, :8].contiguous().view(torch.float32)
    assert int((header == 1).all(1).sum()) == R - at.size


def test_quantized_cache_of_more_threads_than_a_grid_holds():
    # 64 threads a bag of 272 elements: beyond 6.7e7 bags more than 2^32.  A few bags have lookups, at both ends and where one
    # launch ends and the next begins.
    B, D, R, q = 68_000_000, 272, 50, "int8"
    rng = np.random.default_rng(11)
    t = torch.from_numpy(rng.standard_normal((R, D)).astype(np.float32)).to(H.DEV)
    hot = np.arange(0, R, 2, dtype=np.int64)
    cache = torch.empty((hot.size, emb.emb_row_bytes(D, q)), dtype=torch.uint8, device=H.DEV)
    index = torch.empty(emb.emb_cache_index_bytes(R), dtype=torch.uint8, device=H.DEV)
    status, hm = torch.zeros(1, dtype=torch.int32, device=H.DEV), torch.zeros(2, dtype=torch.int64, device=H.DEV)
    emb.emb_cache_build_quantized(t.data_ptr(), R, D, "f32", q, H.dev(hot), cache, index, status)
    bags = np.unique(np.concatenate([np.arange(c, c + 40) for c in (0, (1 << 25) - 20, (1 << 26) - 20, B - 40)]))
    where = torch.from_numpy(bags).to(H.DEV)
    lengths = torch.zeros(B + 1, dtype=torch.int64, device=H.DEV)
    lengths[where + 1] = torch.arange(bags.size, device=H.DEV) % 5
    off = torch.cumsum(lengths, 0)
    rows = rng.integers(0, R, int(off[-1])).astype(np.int64)
    out = torch.full((1, B, D), 9.0, device=H.DEV)
    emb.emb_bag_forward_cached_quantized(t.data_ptr(), R, D, "f32", q, cache, index, hot.size, H.dev(rows), off, B, "sum", out, hm, status)
    vals = t.double().cpu().numpy()
    vals[hot] = mx.int_values(cache.cpu().numpy(), D, q)
    n = np.arange(bags.size) % 5
    ref, mag = mx.pool(vals[rows], np.concatenate(([0], np.cumsum(n))), "sum")
    got = out[0, where].cpu().numpy()
    assert np.all(np.abs(got - ref) <= (n[:, None] + 2) * 2.0 ** -24 * mag)
    hits = int(np.isin(rows, hot).sum())
    assert hm.cpu().tolist() == [hits, rows.size - hits] and status.item() == 0
    used = 0
    for b0 in range(0, B, 1 << 23):                          # every other bag is empty
        used += int(torch.count_nonzero(out[0, b0:b0 + (1 << 23)].any(1)))
    assert used == np.count_nonzero(got.any(1))


@pytest.mark.parametrize("kind", ["mxfp4", "bf16", "f32"])
@pytest.mark.parametrize("M,N,D", [(65, 1_000_000, 64), (65, 1_100_000, 64), (70, 600_000, 96), (129, 700_001, 128)])
def test_product_of_short_rows_on_both_sides_of_the_early_read(M, N, D, kind):
    # W of 38 to 56 MB (its rows are read ahead up to 48 MiB): sums of 4 integers, exact
    rng = np.random.default_rng(N + D)
    codes = torch.randint(0, 16, (N, D // 2, 2), dtype=torch.uint8, device=H.DEV, generator=torch.Generator(H.DEV).manual_seed(N))
    w = torch.zeros((N, emb.emb_row_bytes(D, "mxfp4")), dtype=torch.uint8, device=H.DEV)
    w[:, :D // 2] = codes[:, :, 0] | codes[:, :, 1] << 4
    w[:, D // 2:D // 2 + D // 32] = 128
    values = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float32, device=H.DEV)     # at this scale
    v = (values[(codes & 7).long()] * (1 - 2 * (codes >> 3).float())).reshape(N, D)
    x = torch.zeros((M, D), device=H.DEV)
    at = torch.from_numpy(np.argsort(rng.random((M, D)), 1)[:, :4].copy()).to(H.DEV)
    x.scatter_(1, at, torch.from_numpy(rng.choice([-2.0, -1.0, 1.0, 2.0], (M, 4)).astype(np.float32)).to(H.DEV))
    o = torch.full((M, N), 0.5, device=H.DEV)
    if kind == "mxfp4":
        small = torch.empty((M, w.shape[1]), dtype=torch.uint8, device=H.DEV)
        emb.emb_quantize_rows_from(x, "mxfp4", small)
        emb.emb_rows_product(small, w, D, o)
    else:
        emb.emb_rows_product(x.to(TORCH[kind]), w, D, o)
    for m in range(0, M, 8):
        ref = sum(x[m, k] * v[:, k] for k in at[m].tolist())
        assert torch.equal(o[m], ref), m
    assert not (o == 0.5).any()
