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
