"""MXFP4 rows on the GPU against their definition in 64 bits: quantising and reading back, the pooled lookups, the cache
that is quantised as it is written, the product with the rows, and all of them in a row.

Tolerances.  Quantising, MXFP4 values and copies are exact.  A pooled sum of n rows makes n - 1 fp32 additions of at most
half a step (2^-24) of sum |v|, a mean one division more.  A product makes one addition an element (three an element for
an fp32 x) of at most one step (2^-23) of sum |x||w|, whichever way the matrix unit cuts; its cast to bf16 half a
step (2^-8) of the value."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2508_05700_amd import binding as emb  # noqa: E402
from paper_2508_05700_amd import pipeline  # noqa: E402
from tests import harness as H  # noqa: E402
from tests import mx_plain as mx  # noqa: E402

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def _status():
    return torch.zeros(1, dtype=torch.int32, device=H.DEV)


def _src(rng, R, D, dtype):
    """A matrix of rows of very different size, on the device, and the same in float64."""
    x = rng.standard_normal((R, D)) * 2.0 ** rng.integers(-20, 20, (R, 1))
    t = torch.from_numpy(x.astype(np.float32)).to(TORCH[dtype])
    return t.to(H.DEV), t.double().numpy()


def _special(D, dtype):
    """Rows of values that are easy to get wrong."""
    rows = []
    grid = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 4.0, 0.249, 0.251, 4.99, 5.01, 7.99, 0.0]
    for e in (0, 1, -30, 60, -120, -126, -130, 121):
        v = np.array(grid + [-g for g in grid]) * 2.0 ** e
        rows.append(np.resize(v, D))
    rows.append(np.zeros(D))
    rows.append(np.full(D, -0.0))
    rows.append(np.full(D, 3.3e38))
    for bad in (np.nan, np.inf, -np.inf):       # in one block only
        v = np.ones(D)
        v[D // 2 // 32 * 32 + 5] = bad
        rows.append(v)
    with np.errstate(over="ignore"):
        t = torch.from_numpy(np.array(rows).astype(np.float32)).to(TORCH[dtype])
    return t.to(H.DEV), t.double().numpy()


# ---------------------------------------------------------------------------
# quantising and reading back
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,D", [(1, 32), (3, 64), (130, 96), (77, 128), (5, 1056), (2, 4096), (1, 65536), (301, 32), (33, 256)])
def test_quantize_is_the_definition_byte_for_byte(R, D, dtype):
    rng = np.random.default_rng(R + D)
    for t, x in (_src(rng, R, D, dtype), _special(min(D, 1056), dtype)):
        n, d = x.shape
        want = mx.pack(*mx.quantize(x))
        for pad in (0, 16):                     # rows next to each other, and apart
            src = torch.full((n, d + pad), 1e30, dtype=t.dtype, device=H.DEV)
            src[:, :d] = t
            out = torch.full((n + 2, want.shape[1]), 0xA5, dtype=torch.uint8, device=H.DEV)
            emb.emb_quantize_rows_from(src[:, :d], "mxfp4", out[1:n + 1])
            got = out.cpu().numpy()
            assert np.array_equal(got[1:n + 1], want), (n, d, pad)
            assert (got[[0, n + 1]] == 0xA5).all()
        if dtype == "f32":
            out = torch.empty((n, want.shape[1]), dtype=torch.uint8, device=H.DEV)
            emb.emb_quantize_rows(t.contiguous(), "mxfp4", out)
            assert np.array_equal(out.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,D", [(1, 32), (130, 96), (5, 1056), (3, 4096), (301, 64)])
def test_rows_read_back(R, D, dtype):
    rng = np.random.default_rng(R * D)
    rows = mx.random_rows(rng, R, D, 0, 255)
    rows[0, D // 2] = 255
    rows[R // 2, D // 2 + D // 32 - 1] = 254
    want = torch.from_numpy(mx.values(rows, D)).to(torch.float32)
    want = want.to(TORCH[dtype])                # exact: two bits of significand
    out = torch.full((R, D + 16), 7.0, dtype=TORCH[dtype], device=H.DEV)
    emb.emb_dequantize_rows(H.dev(rows), "mxfp4", out[:, :D])
    got = out.cpu()
    assert torch.equal(got[:, :D].isnan(), want.isnan())
    assert torch.equal(got[:, :D].nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
    assert (got[:, D:] == 7.0).all()


@pytest.mark.parametrize("q", ["int8", "int4", "int4r64"])
@pytest.mark.parametrize("D", [16, 48, 128, 1024])
def test_int_rows_from_bf16_and_strided_rows_and_back(D, q):
    rng = np.random.default_rng(D)
    R = 37
    t, _ = _src(rng, R, D + 16, "bf16")
    t = t[:, 16:]
    rb = emb.emb_row_bytes(D, q)
    a, b = (torch.empty((R, rb), dtype=torch.uint8, device=H.DEV) for _ in range(2))
    emb.emb_quantize_rows_from(t, q, a)
    emb.emb_quantize_rows(t.float().contiguous(), q, b)
    assert torch.equal(a, b)
    want = mx.int_values(a.cpu().numpy(), D, q)
    for dtype, half in (("f32", 2.0 ** -24), ("bf16", 2.0 ** -8)):
        out = torch.full((R, D + 8), 5.0, dtype=TORCH[dtype], device=H.DEV)
        emb.emb_dequantize_rows(a, q, out[:, :D])
        got = out.cpu().double().numpy()
        # one fused multiply-add (half a step of fp32), then for bf16 half a step of that
        assert np.all(np.abs(got[:, :D] - want) <= (half + 2.0 ** -24) * np.abs(want))
        assert (got[:, D:] == 5.0).all()


def test_rows_beyond_32_bit_offsets():
    # 1.4e8 rows of 32 bytes: the last ones stand beyond 2^32 bytes, and so do their bf16 values
    R, D, k = 140_000_000, 32, 1000
    rng = np.random.default_rng(3)
    t, x = _src(rng, k, D, "bf16")
    src = torch.zeros((R, D), dtype=torch.bfloat16, device=H.DEV)
    src[-k:] = t
    rows = torch.empty((R, 32), dtype=torch.uint8, device=H.DEV)
    emb.emb_quantize_rows_from(src, "mxfp4", rows)
    want = mx.pack(*mx.quantize(x))
    assert np.array_equal(rows[-k:].cpu().numpy(), want)
    src.fill_(1.0)
    emb.emb_dequantize_rows(rows, "mxfp4", src)
    assert torch.equal(src[-k:].cpu(), torch.from_numpy(mx.values(want, D)).to(torch.bfloat16))
    assert not src[:1000].any()
    del src
    ids = torch.from_numpy(np.array([R - 1, R - k, 0, R - 2], dtype=np.int64)).to(H.DEV)
    out = torch.empty((1, 2, D), dtype=torch.float32, device=H.DEV)
    emb.emb_bag_forward(emb.TableSet([rows], D, "mxfp4"), ids, H.dev(np.array([0, 3, 4], dtype=np.int64)), 2, "sum", out)
    v = mx.values(want, D)
    assert np.allclose(out.cpu().numpy()[0], np.stack((v[-1] + v[0], v[-2])), rtol=2.0 ** -23, atol=0)
    scores = torch.empty((1, R), dtype=torch.float32, device=H.DEV)
    emb.emb_rows_product(torch.ones((1, D), dtype=torch.bfloat16, device=H.DEV), rows, D, scores)
    got = scores[0, -k:].cpu().double().numpy()
    assert np.all(np.abs(got - v.sum(1)) <= D * 2.0 ** -23 * np.abs(v).sum(1))
    assert not scores[0, :1000].any()


# ---------------------------------------------------------------------------
# pooled lookups
# ---------------------------------------------------------------------------
def _batch(rng, T, B, R, max_len):
    lengths = rng.integers(0, max_len + 1, size=T * B).astype(np.int32)
    lengths[rng.integers(0, T * B, size=max(1, T * B // 5))] = 0
    off = np.zeros(T * B + 1, dtype=np.int64)
    np.cumsum(lengths, out=off[1:])
    return lengths, off, rng.integers(0, R, size=int(off[-1])).astype(np.int64)


def _check_pool(got, tables, rows, off, B, mode):
    for t, v in enumerate(tables):
        ref, mag = mx.pool(v[rows[off[t * B]:off[(t + 1) * B]]], off[t * B:(t + 1) * B + 1] - off[t * B], mode)
        n = (off[t * B + 1:(t + 1) * B + 1] - off[t * B:(t + 1) * B])[:, None]
        assert np.all(np.abs(got[t] - ref) <= (n + 1) * 2.0 ** -24 * mag)
        assert (got[t][n[:, 0] == 0] == 0).all()


@pytest.mark.parametrize("mode", ["sum", "mean"])
@pytest.mark.parametrize("T,B,R,D,max_len", [(1, 1, 1, 32, 1), (2, 9, 50, 64, 40), (3, 70, 200, 96, 9), (1, 33, 100, 128, 70),
                                             (2, 5, 64, 320, 20), (1, 3, 90, 1024, 300), (5, 40, 30, 32, 3)])
def test_lookups_over_mxfp4_rows(T, B, R, D, max_len, mode):
    rng = np.random.default_rng(T * B + D)
    packed = [mx.random_rows(rng, R, D) for _ in range(T)]
    vals = [mx.values(p, D) for p in packed]
    lengths, off, rows = _batch(rng, T, B, R, max_len)
    ts = emb.TableSet([H.dev(p) for p in packed], D, "mxfp4")
    out = torch.full((T, B, D), 9.0, dtype=torch.float32, device=H.DEV)
    st = _status()
    emb.emb_bag_forward(ts, H.dev(rows), H.dev(off), B, mode, out, st)
    first = out.cpu().numpy()
    assert st.item() == 0
    _check_pool(first, vals, rows, off, B, mode)
    # from bag lengths: the same bits
    off_out = torch.empty(T * B + 1, dtype=torch.int64, device=H.DEV)
    scratch = torch.empty(emb.emb_offsets_scratch_bytes(T * B), dtype=torch.uint8, device=H.DEV)
    out.fill_(9.0)
    emb.emb_bag_forward_lengths(ts, H.dev(rows), H.dev(lengths), B, mode, out, off_out, scratch, st)
    assert np.array_equal(out.cpu().numpy(), first) and np.array_equal(off_out.cpu().numpy(), off)
    # from raw IDs: those whose rows come back
    raw = rng.integers(0, 1 << 63, size=rows.size, dtype=np.int64)
    got_rows = torch.empty(rows.size, dtype=torch.int64, device=H.DEV)
    emb.emb_bag_forward_hashed(ts, H.dev(raw), H.dev(off), B, mode, out, got_rows, st)
    _check_pool(out.cpu().numpy(), vals, got_rows.cpu().numpy(), off, B, mode)
    # a hosted table of such rows, cached in its own type, alone and in a set, and its misses fetched ahead
    hot = np.sort(rng.choice(R, size=max(1, R // 4), replace=False)).astype(np.int64)
    p = H.dev(packed[0])
    cache = torch.empty((hot.size, p.shape[1]), dtype=torch.uint8, device=H.DEV)
    index = torch.empty(emb.emb_cache_index_bytes(R), dtype=torch.uint8, device=H.DEV)
    emb.emb_cache_build(p.data_ptr(), R, D, "mxfp4", H.dev(hot), cache, index, st)
    n0 = int(off[B])
    r0, o0 = H.dev(rows[:n0]), H.dev(off[:B + 1])
    one = torch.full((1, B, D), 9.0, dtype=torch.float32, device=H.DEV)
    emb.emb_bag_forward_cached(p.data_ptr(), R, D, "mxfp4", cache, index, hot.size, r0, o0, B, mode, one, None, st)
    assert np.array_equal(one.cpu().numpy()[0], first[0])
    ct = emb.CachedTables([(p.data_ptr(), R, cache, index, hot.size, 0)], D, "mxfp4")
    one.fill_(9.0)
    emb.emb_bag_forward_cached_tables(ct, r0, o0, B, mode, one, None, st)
    assert np.array_equal(one.cpu().numpy()[0], first[0])
    loc = torch.empty(max(n0, 1), dtype=torch.int64, device=H.DEV)
    stage = torch.empty((max(n0, 1), p.shape[1]), dtype=torch.uint8, device=H.DEV)
    count = torch.zeros(1, dtype=torch.int64, device=H.DEV)
    emb.emb_cache_stage_misses(p.data_ptr(), R, D, "mxfp4", index, hot.size, r0, stage, max(n0 // 2, 1), loc, count, st)
    one.fill_(9.0)
    emb.emb_bag_forward_staged(p.data_ptr(), R, D, "mxfp4", cache, hot.size, stage, max(n0 // 2, 1), loc[:n0], o0, B, mode, one, None, st)
    assert np.array_equal(one.cpu().numpy()[0], first[0])
    assert st.item() == 0


def test_versions_refresh_and_bag_lengths_of_hosted_mxfp4_tables():
    # the remaining lookups that take the type: latched tables, hosted sets from bag lengths, and a policy-run cache of its own type
    rng = np.random.default_rng(12)
    T, R, D, B = 2, 300, 96, 37
    packed = [mx.random_rows(rng, R, D) for _ in range(T)]
    vals = [mx.values(p, D) for p in packed]
    dev = [H.dev(p) for p in packed]
    lengths, off, _ = _batch(rng, T, B, R, 15)
    raw = rng.integers(0, 1 << 63, size=int(off[-1]), dtype=np.int64)
    ts = emb.TableSet(dev, D, "mxfp4", salts=[5, 6])
    st = _status()
    rows, out = torch.empty(raw.size, dtype=torch.int64, device=H.DEV), torch.empty((T, B, D), device=H.DEV)
    off_out = torch.empty(T * B + 1, dtype=torch.int64, device=H.DEV)
    scratch = torch.empty(emb.emb_offsets_scratch_bytes(T * B), dtype=torch.uint8, device=H.DEV)
    emb.emb_bag_forward_hashed_lengths(ts, H.dev(raw), H.dev(lengths), B, "mean", out, off_out, scratch, rows, st)
    first = out.cpu().numpy()
    _check_pool(first, vals, rows.cpu().numpy(), off, B, "mean")
    handle = torch.zeros(1, dtype=torch.int64, device=H.DEV)
    record = torch.empty(emb.emb_version_record_bytes(T), dtype=torch.uint8, device=H.DEV)
    latch = torch.empty(emb.emb_version_latch_bytes(T), dtype=torch.uint8, device=H.DEV)
    emb.emb_version_record_write(record, ts, 3)
    emb.emb_version_publish(handle, record)
    emb.emb_version_latch(handle, T, latch, st)
    out.fill_(9.0)
    emb.emb_bag_forward_latched_hashed(latch, T, D, "mxfp4", H.dev(raw), H.dev(off), B, "mean", out, st)
    assert np.array_equal(out.cpu().numpy(), first)
    caches = [pipeline.HotRowCache(dev[t].data_ptr(), R, D, "mxfp4", 40, 5 + t, torch.device(H.DEV)) for t in range(T)]
    hosted = pipeline.HostedTableSet(caches, torch.device(H.DEV))
    for _ in range(2):
        out.fill_(9.0)
        emb.emb_bag_forward_cached_tables_hashed_lengths(hosted.tables, H.dev(raw), H.dev(lengths), B, "mean", out, off_out, scratch,
                                                         None, st)
        assert np.array_equal(out.cpu().numpy(), first)
        hosted.observe(H.dev(raw), off, B)
        hosted.refresh()
    assert st.item() == 0 and all(c.status.item() == 0 for c in caches)


def test_batches_without_lookups():
    R, D, B = 50, 64, 3
    packed = mx.random_rows(np.random.default_rng(1), R, D)
    none, off = torch.empty(0, dtype=torch.int64, device=H.DEV), torch.zeros(B + 1, dtype=torch.int64, device=H.DEV)
    out = torch.full((1, B, D), 9.0, device=H.DEV)
    emb.emb_bag_forward(emb.TableSet([H.dev(packed)], D, "mxfp4"), none, off, B, "mean", out)
    assert not out.any()
    t = torch.ones((R, D), device=H.DEV)
    index = torch.empty(emb.emb_cache_index_bytes(R), dtype=torch.uint8, device=H.DEV)
    cache = torch.empty((1, 48), dtype=torch.uint8, device=H.DEV)
    emb.emb_cache_build_quantized(t.data_ptr(), R, D, "f32", "mxfp4", none, cache, index)
    out.fill_(9.0)
    emb.emb_bag_forward_cached_quantized(t.data_ptr(), R, D, "f32", "mxfp4", cache, index, 0, none, off, B, "mean", out)
    assert not out.any()
    emb.emb_quantize_rows_from(t[:0], "mxfp4", cache[:0])
    emb.emb_dequantize_rows(cache[:0], "mxfp4", t[:0])
    emb.emb_rows_product(t[:0], cache, D, torch.empty((0, 1), device=H.DEV))
    emb.emb_rows_product(t, cache[:0], D, torch.empty((R, 0), device=H.DEV))


def test_lookups_skip_bad_rows_and_bags_and_pass_on_nan():
    rng = np.random.default_rng(5)
    R, D, B = 40, 64, 5
    packed = mx.random_rows(rng, R, D)
    packed[7, D // 2 + 1] = 255
    v = mx.values(packed, D)
    ts = emb.TableSet([H.dev(packed)], D, "mxfp4")
    rows = np.array([3, -1, 4, 40, 7, 9, 1 << 40], dtype=np.int64)
    off = np.array([0, 2, 4, 5, 6, 7], dtype=np.int64)
    st = _status()
    out = torch.empty((1, B, D), dtype=torch.float32, device=H.DEV)
    emb.emb_bag_forward(ts, H.dev(rows), H.dev(off), B, "sum", out, st)
    got = out.cpu().numpy()[0]
    assert st.item() == emb.STATUS_BAD_INDEX
    assert np.array_equal(got[0], v[3]) and np.array_equal(got[1], v[4]) and np.array_equal(got[3], v[9]) and not got[4].any()
    assert np.isnan(got[2, 32:]).all() and np.array_equal(got[2, :32], v[7, :32])
    st.zero_()
    emb.emb_bag_forward(ts, H.dev(rows[:5]), H.dev(np.array([0, 1, 0, 9, 3, 5], dtype=np.int64)), B, "sum", out, st)
    assert st.item() & emb.STATUS_BAD_OFFSETS and np.array_equal(out.cpu().numpy()[0, 0], v[3])


# ---------------------------------------------------------------------------
# a cache of fewer bits than its table
# ---------------------------------------------------------------------------
def _packed_values(rows, D, q):
    return mx.values(rows, D) if q == "mxfp4" else mx.int_values(rows, D, q)


@pytest.mark.parametrize("mode", ["sum", "mean"])
@pytest.mark.parametrize("q", ["mxfp4", "int8", "int4", "int4r64"])
@pytest.mark.parametrize("dtype,D,R,B,max_len", [("f32", 64, 500, 40, 30), ("bf16", 96, 130, 19, 50), ("f32", 1024, 70, 4, 90),
                                                 ("bf16", 32, 64, 300, 3), ("f32", 32, 1, 1, 1), ("bf16", 512, 65, 7, 11)])
def test_quantized_cache(dtype, D, R, B, max_len, q, mode):
    rng = np.random.default_rng(D + R)
    t, x = _src(rng, R, D, dtype)
    rb = emb.emb_row_bytes(D, q)
    all_rows = torch.empty((R, rb), dtype=torch.uint8, device=H.DEV)
    emb.emb_quantize_rows_from(t, q, all_rows)
    packed = all_rows.cpu().numpy()
    _, off, rows = _batch(rng, 1, B, R, max_len)
    ptr = t.data_ptr()
    for num_hot in sorted({0, 1, R // 3, R}):
        hot = np.sort(rng.choice(R, size=num_hot, replace=False)).astype(np.int64)
        st, hm = _status(), torch.zeros(2, dtype=torch.int64, device=H.DEV)
        cache = torch.full((num_hot + 1, rb), 0xA5, dtype=torch.uint8, device=H.DEV)
        index = torch.full((emb.emb_cache_index_bytes(R),), 0xA5, dtype=torch.uint8, device=H.DEV)
        emb.emb_cache_build_quantized(ptr, R, D, dtype, q, H.dev(hot), cache, index, st)
        got = cache.cpu().numpy()
        assert np.array_equal(got[:num_hot], packed[hot]) and (got[num_hot] == 0xA5).all()
        vals = x.copy()
        vals[hot] = _packed_values(packed, D, q)[hot]
        out = torch.full((1, B, D), 9.0, dtype=torch.float32, device=H.DEV)
        emb.emb_bag_forward_cached_quantized(ptr, R, D, dtype, q, cache, index, num_hot, H.dev(rows), H.dev(off), B, mode, out, hm, st)
        ref, mag = mx.pool(vals[rows], off, mode)
        n = np.diff(off)[:, None]
        # INT rows: one fused multiply-add a value more
        assert np.all(np.abs(out.cpu().numpy()[0] - ref) <= (n + 2) * 2.0 ** -24 * mag)
        hits = int(np.isin(rows, hot).sum())
        assert hm.cpu().tolist() == [hits, rows.size - hits] and st.item() == 0
        # refreshed from an older cache that holds half of the rows: the same bytes
        old = hot[::2]
        other = np.setdiff1d(np.arange(R), hot)[:5]
        old = np.sort(np.concatenate((old, other))).astype(np.int64)
        oc = torch.empty((max(old.size, 1), rb), dtype=torch.uint8, device=H.DEV)
        oi, ni = torch.empty_like(index), torch.empty_like(index)
        emb.emb_cache_build_quantized(ptr, R, D, dtype, q, H.dev(old), oc, oi, st)
        oc2 = oc.clone()
        oc2[:, 0] ^= 1                           # told apart: a kept row is a copy, not made again
        nc = torch.full((num_hot + 1, rb), 0xA5, dtype=torch.uint8, device=H.DEV)
        moved = torch.zeros(2, dtype=torch.int64, device=H.DEV)
        emb.emb_cache_rebuild_quantized(ptr, R, D, dtype, q, oc2, oi, old.size, H.dev(hot), nc, ni, moved, st)
        kept = np.isin(hot, old)
        want = packed[hot].copy()
        want[kept, 0] ^= 1
        got = nc.cpu().numpy()
        assert np.array_equal(got[:num_hot], want) and (got[num_hot] == 0xA5).all() and torch.equal(ni, index)
        assert moved.cpu().tolist() == [int(kept.sum()), int((~kept).sum())] and st.item() == 0


def test_quantized_cache_bad_rows_and_hot_sets():
    rng = np.random.default_rng(17)
    R, D, B = 100, 64, 4
    t, x = _src(rng, R, D, "f32")
    st = _status()
    index = torch.empty(emb.emb_cache_index_bytes(R), dtype=torch.uint8, device=H.DEV)
    cache = torch.full((4, emb.emb_row_bytes(D, "mxfp4")), 0xA5, dtype=torch.uint8, device=H.DEV)
    emb.emb_cache_build_quantized(t.data_ptr(), R, D, "f32", "mxfp4", H.dev(np.array([5, -1, 100, 7], dtype=np.int64)), cache, index, st)
    assert st.item() == emb.STATUS_BAD_HOT_SET
    got = cache.cpu().numpy()
    want = mx.pack(*mx.quantize(x))
    assert np.array_equal(got[[0, 3]], want[[5, 7]]) and (got[1:3] == 0xA5).all()
    st.zero_()
    hot = np.array([1, 2, 3], dtype=np.int64)
    emb.emb_cache_build_quantized(t.data_ptr(), R, D, "f32", "mxfp4", H.dev(hot), cache, index, st)
    vals = x.copy()
    vals[hot] = mx.values(want, D)[hot]
    out = torch.empty((1, B, D), dtype=torch.float32, device=H.DEV)
    hm = torch.zeros(2, dtype=torch.int64, device=H.DEV)
    rows = np.array([1, 50, -3, 2, 100, 60, 3], dtype=np.int64)
    emb.emb_bag_forward_cached_quantized(t.data_ptr(), R, D, "f32", "mxfp4", cache, index, 3, H.dev(rows),
                                         H.dev(np.array([0, 2, 3, 7, 7], dtype=np.int64)), B, "sum", out, hm, st)
    assert st.item() == emb.STATUS_BAD_INDEX and hm.cpu().tolist() == [3, 2]
    got = out.cpu().numpy()[0]
    assert np.allclose(got[0], vals[1] + vals[50], rtol=2.0 ** -23, atol=2.0 ** -23 * np.abs(vals[[1, 50]]).max())
    assert not got[1].any() and not got[3].any()
    st.zero_()
    emb.emb_bag_forward_cached_quantized(t.data_ptr(), R, D, "f32", "mxfp4", cache, index, 3, H.dev(rows[:2]),
                                         H.dev(np.array([0, 1, 0, 5, 2], dtype=np.int64)), B, "sum", out, hm, st)
    assert st.item() & emb.STATUS_BAD_OFFSETS and np.array_equal(out.cpu().numpy()[0, 0], vals[1].astype(np.float32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_hot_row_cache_in_fewer_bits_over_a_host_table(dtype):
    # watched, refreshed twice, looked up by raw IDs; the table stands in pinned host memory
    rng = np.random.default_rng(23)
    R, D, B = 3000, 64, 200
    t, x = _src(rng, R, D, dtype)
    host = t.cpu().pin_memory()
    ptr = emb.emb_host_device_pointer(int(host.data_ptr()))
    c = pipeline.HotRowCache(ptr, R, D, dtype, 300, 77, torch.device(H.DEV), cache_dtype="mxfp4")
    q = mx.values(mx.pack(*mx.quantize(x)), D)
    raw = (rng.zipf(1.2, size=6000) % 100_000).astype(np.int64)
    raw_dev, rows = H.dev(raw), torch.empty(raw.size, dtype=torch.int64, device=H.DEV)
    emb.emb_hash_ids(raw_dev, 77, R, rows)
    rows = rows.cpu().numpy()
    off = np.sort(np.concatenate(([0, raw.size], rng.integers(0, raw.size + 1, size=B - 1)))).astype(np.int64)
    for _ in range(3):
        out = torch.empty((1, B, D), dtype=torch.float32, device=H.DEV)
        c.hit_miss.zero_()
        c.forward_hashed(raw_dev, H.dev(off), B, "mean", out)
        hot = c.hot[:c.num_hot].cpu().numpy()
        vals = x.copy()
        vals[hot] = q[hot]
        ref, mag = mx.pool(vals[rows], off, "mean")
        n = np.diff(off)[:, None]
        assert np.all(np.abs(out.cpu().numpy()[0] - ref) <= (n + 2) * 2.0 ** -24 * mag)
        hits = int(np.isin(rows, hot).sum())
        assert c.hit_miss.cpu().tolist() == [hits, rows.size - hits]
        c.observe(raw_dev)
        c.refresh()
    assert c.status.item() == 0 and hits > rows.size // 3
    with pytest.raises(AssertionError):
        pipeline.HostedTableSet([c], torch.device(H.DEV))


# ---------------------------------------------------------------------------
# the product
# ---------------------------------------------------------------------------
def _operand(rng, M, D, kind, pad=0):
    """A device operand of M rows and its float64 values."""
    if kind == "mxfp4":
        rows = mx.random_rows(rng, M, D, 120, 131)
        return H.dev(rows), mx.values(rows, D)
    x = rng.standard_normal((M, D)) * 2.0 ** rng.integers(-3, 4, (M, 1))
    t = torch.from_numpy(x.astype(np.float32)).to(TORCH[kind])
    wide = torch.full((M, D + pad), float("nan"), dtype=t.dtype, device=H.DEV)
    wide[:, :D] = t.to(H.DEV)
    return wide[:, :D], t.double().numpy()


def _check_product(got, x, w, kind, out):
    ref = x @ w.T
    mag = np.abs(x) @ np.abs(w).T
    D = x.shape[1]
    tol = D * (3 if kind == "f32" else 1) * 2.0 ** -23 * mag
    if out == "bf16":
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5].tolist(), got[bad][:5], ref[bad][:5])


SHAPES = [(1, 1, 32), (1, 1000, 64), (1, 37, 2048), (2, 17, 96), (15, 64, 128), (16, 257, 160), (17, 16, 512), (31, 100, 544),
          (33, 130, 1056), (64, 63, 32), (65, 4, 64), (100, 513, 64), (129, 255, 320), (257, 300, 4096), (300, 1, 128), (5, 700, 16384),
          (512, 512, 1024), (30, 90, 96), (60, 70_000, 96), (50, 66_000, 1024), (20, 50_001, 256)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["mxfp4", "bf16", "f32"])
@pytest.mark.parametrize("M,N,D", SHAPES)
def test_product(M, N, D, kind, out):
    rng = np.random.default_rng(M * 7 + N * 3 + D)
    w = mx.random_rows(rng, N, D, 118, 129)
    x, xv = _operand(rng, M, D, kind, pad=16)
    wv = mx.values(w, D)
    for pad in (0, 3):                       # rows of the output apart, and not on 16 bytes
        o = torch.full((M, N + pad), 3.0, dtype=TORCH[out], device=H.DEV)
        emb.emb_rows_product(x, H.dev(w), D, o[:, :N])
        got = o.cpu().double().numpy()
        _check_product(got[:, :N], xv, wv, kind, out)
        assert (got[:, N:] == 3.0).all()


@pytest.mark.parametrize("kind", ["mxfp4", "bf16", "f32"])
@pytest.mark.parametrize("M,N,D", [(4100, 4203, 288), (4500, 4096, 544), (300, 66_000, 160), (8193, 2100, 96)])
def test_product_of_many_tiles(M, N, D, kind):
    # enough tiles of the largest kind, an odd and an even number of stages, edges both ways
    rng = np.random.default_rng(M + N)
    w = mx.random_rows(rng, N, D, 118, 129)
    x, xv = _operand(rng, M, D, kind)
    o = torch.full((M, N), float("nan"), dtype=torch.float32, device=H.DEV)
    emb.emb_rows_product(x, H.dev(w), D, o)
    got, wv = o.cpu().numpy(), mx.values(w, D)
    for rows in (np.arange(0, M, 97), np.arange(M - 140, M)):
        _check_product(got[rows].astype(np.float64), xv[rows], wv, kind, "f32")
    cols = np.concatenate((np.arange(0, N, 101), np.arange(N - 70, N)))
    _check_product(got[:, cols].astype(np.float64), xv, wv[cols], kind, "f32")
    assert not np.isnan(got).any()


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["mxfp4", "bf16", "f32"])
@pytest.mark.parametrize("M,N,D", [(4099, 4096, 1056), (1054, 8190, 1024), (513, 16_300, 1504), (288, 32_768, 1024)])
def test_product_of_a_few_rows_past_whole_tiles(M, N, D, kind, out):
    rng = np.random.default_rng(M + N + D)
    w = mx.random_rows(rng, N, D, 118, 129)
    x, xv = _operand(rng, M, D, kind, pad=8)
    o = torch.full((M + 1, N + 5), 3.0, dtype=TORCH[out], device=H.DEV)
    emb.emb_rows_product(x, H.dev(w), D, o[:M, :N])
    got, wv = o.cpu().float().numpy(), mx.values(w, D)
    assert (got[M] == 3.0).all() and (got[:, N:] == 3.0).all()
    for rows in (np.arange(0, M, 193), np.arange(M - 40, M)):
        _check_product(got[rows, :N].astype(np.float64), xv[rows], wv, kind, out)
    cols = np.concatenate((np.arange(0, N, 401), np.arange(N - 20, N)))
    _check_product(got[:M, cols].astype(np.float64), xv, wv[cols], kind, out)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_product_of_rows_very_far_apart(kind):
    M, N, D, stride = 40, 70, 64, 3 << 20          # more than 4 MB from row to row
    rng = np.random.default_rng(8)
    x, xv = _operand(rng, M, D, kind)
    far = torch.full((M, stride), float("nan"), dtype=x.dtype, device=H.DEV)
    far[:, :D] = x
    w = mx.random_rows(rng, N, D, 118, 129)
    o = torch.empty((M, N), dtype=torch.float32, device=H.DEV)
    emb.emb_rows_product(far[:, :D], H.dev(w), D, o)
    _check_product(o.cpu().double().numpy(), xv, mx.values(w, D), kind, "f32")


@pytest.mark.parametrize("kind", ["mxfp4", "bf16", "f32"])
@pytest.mark.parametrize("M,N,D", [(3, 40, 96), (70, 150, 288), (300, 280, 64)])
def test_product_passes_on_nan_and_infinity(M, N, D, kind):
    rng = np.random.default_rng(M + D)
    w = mx.random_rows(rng, N, D, 118, 129)
    wv = mx.values(w, D)
    w[N // 2, D // 2 + D // 32 - 1] = 255
    x, xv = _operand(rng, M, D, kind)
    o = torch.empty((M, N), dtype=torch.float32, device=H.DEV)
    emb.emb_rows_product(x, H.dev(w), D, o)
    got = o.cpu().double().numpy()
    assert np.isnan(got[:, N // 2]).all()
    keep = np.arange(N) != N // 2
    _check_product(got[:, keep], xv, wv[keep], kind, "f32")
    w[N // 2, D // 2 + D // 32 - 1] = 120
    if kind == "mxfp4":
        x[M // 2, D // 2] = 255
    else:
        x = x.clone()
        x[M // 2, 5] = float("inf")
        x[0, 3] = float("nan")
        nan_low = torch.tensor([0x7F800001], dtype=torch.int32).view(torch.float32)   # a NaN whose mark is in the lower half
        if kind == "f32":
            x[M - 1, 1] = nan_low.to(H.DEV)[0]
    w[:, :D // 2] |= 0x11                     # no zeros for an infinity to meet
    wv = mx.values(w, D)
    emb.emb_rows_product(x, H.dev(w), D, o)
    got = o.cpu().numpy()
    if kind == "mxfp4":
        assert np.isnan(got[M // 2]).all() and np.isfinite(np.delete(got, M // 2, 0)).all()
    else:
        assert np.isnan(got[0]).all()
        assert np.array_equal(got[M // 2], np.where(wv[:, 5] > 0, np.inf, -np.inf).astype(np.float32))
        if kind == "f32":
            assert np.isnan(got[M - 1]).all()


def test_product_of_extreme_scales():
    rng = np.random.default_rng(2)
    D = 64
    for sw, sx in ((0, 254), (254, 3), (1, 200), (250, 0), (130, 120)):
        w, x = mx.random_rows(rng, 40, D, sw, sw + 1), mx.random_rows(rng, 20, D, sx, sx + 1)
        o = torch.empty((20, 40), dtype=torch.float32, device=H.DEV)
        emb.emb_rows_product(H.dev(x), H.dev(w), D, o)
        _check_product(o.cpu().double().numpy(), mx.values(x, D), mx.values(w, D), "mxfp4", "f32")
        xb = torch.from_numpy(mx.values(x, D).astype(np.float32)).to(torch.bfloat16)
        if sx < 254 and sw < 253:
            emb.emb_rows_product(xb.to(H.DEV), H.dev(w), D, o)
            _check_product(o.cpu().double().numpy(), xb.double().numpy(), mx.values(w, D), "bf16", "f32")


def test_product_of_fp32_keeps_all_of_its_bits():
    # values whose last bits decide: x = 1 + 2^-23 times rows that cancel the 1
    D = 64
    w = np.zeros((1, D // 2), dtype=np.uint8)
    w[0, :16] = 0x22          # +1
    w[0, 16:] = 0xAA          # -1
    rows = np.concatenate((w, np.full((1, 2), 127, dtype=np.uint8), np.zeros((1, 14), dtype=np.uint8)), 1)
    x = np.ones((1, D), dtype=np.float32)
    x[0, :32] += np.float32(2.0 ** -23)
    o = torch.empty((1, 1), dtype=torch.float32, device=H.DEV)
    emb.emb_rows_product(H.dev(x), H.dev(rows), D, o)
    assert o.item() == 32 * 2.0 ** -23


def test_product_with_outputs_beyond_32_bits():
    M, N, D = 33_000, 70_000, 32       # 2.3e9 outputs
    rng = np.random.default_rng(4)
    w = mx.random_rows(rng, N, D, 120, 127)
    x, xv = _operand(rng, M, D, "bf16")
    o = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device=H.DEV)
    emb.emb_rows_product(x, H.dev(w), D, o)
    wv = mx.values(w, D)
    for m in (0, 1, M // 2, M - 2, M - 1):
        _check_product(o[m:m + 1].cpu().double().numpy(), xv[m:m + 1], wv, "bf16", "bf16")
    assert not o[::997].isnan().any()


def test_binding_refuses_shapes_that_do_not_fit():
    w = torch.zeros((8, 48), dtype=torch.uint8, device=H.DEV)
    x = torch.zeros((4, 64), device=H.DEV)
    o = torch.zeros((4, 8), device=H.DEV)
    emb.emb_rows_product(x, w, 64, o)
    for bad in (lambda: emb.emb_rows_product(x[:, :32], w, 64, o), lambda: emb.emb_rows_product(x, w[:7], 64, o),
                lambda: emb.emb_rows_product(x, w, 64, o[:3]), lambda: emb.emb_rows_product(x.double(), w, 64, o),
                lambda: emb.emb_rows_product(x.t(), w, 64, o), lambda: emb.emb_rows_product(x, w, 64, o.t()),
                lambda: emb.emb_rows_product(x.cpu(), w, 64, o), lambda: emb.emb_quantize_rows_from(x, "mxfp4", w),
                lambda: emb.emb_quantize_rows_from(x.half(), "mxfp4", w[:4]), lambda: emb.emb_dequantize_rows(w, "mxfp4", x)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(emb.EmbError):
        emb.emb_quantize_rows_from(torch.zeros((4, 66), device=H.DEV)[:, :64], "mxfp4", w[:4])     # rows not on 16 bytes


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
def test_train_quantize_look_up_and_score():
    # one step of training, the table stored in 4 bits, looked up, and the pooled rows scored against the table's own rows
    rng = np.random.default_rng(31)
    R, D, B = 700, 64, 50
    t, _ = _src(rng, R, D, "bf16")
    t *= 2.0 ** -8
    acc = torch.zeros(R, dtype=torch.float32, device=H.DEV)
    ts = emb.TableSet([t], D, "bf16", [acc])
    _, off, rows = _batch(rng, 1, B, R, 12)
    ws = torch.empty(emb.emb_bag_backward_workspace_bytes(1, B, rows.size, R, D, "bf16"), dtype=torch.uint8, device=H.DEV)
    dout = torch.randn((1, B, D), device=H.DEV)
    emb.emb_bag_backward_rowwise_adagrad(ts, H.dev(rows), H.dev(off), B, "sum", dout, 0.05, 1e-8, ws)
    packed = torch.empty((R, emb.emb_row_bytes(D, "mxfp4")), dtype=torch.uint8, device=H.DEV)
    emb.emb_quantize_rows_from(t, "mxfp4", packed)
    want = mx.pack(*mx.quantize(t.cpu().double().numpy()))
    assert np.array_equal(packed.cpu().numpy(), want)
    pooled = torch.empty((1, B, D), dtype=torch.float32, device=H.DEV)
    emb.emb_bag_forward(emb.TableSet([packed], D, "mxfp4"), H.dev(rows), H.dev(off), B, "mean", pooled)
    v = mx.values(want, D)
    _check_pool(pooled.cpu().numpy(), [v], rows, off, B, "mean")
    scores = torch.empty((B, R), dtype=torch.float32, device=H.DEV)
    emb.emb_rows_product(pooled[0], packed, D, scores)
    p = pooled[0].cpu().double().numpy()
    _check_product(scores.cpu().double().numpy(), p, v, "f32", "f32")
    small = torch.empty((B, packed.shape[1]), dtype=torch.uint8, device=H.DEV)
    emb.emb_quantize_rows_from(pooled[0], "mxfp4", small)
    emb.emb_rows_product(small, packed, D, scores)
    _check_product(scores.cpu().double().numpy(), mx.values(mx.pack(*mx.quantize(p)), D), v, "mxfp4", "f32")


def test_captured_in_a_graph_and_replayed_on_new_inputs():
    rng = np.random.default_rng(41)
    R, D, B, M = 900, 128, 64, 40
    t, x = _src(rng, R, D, "f32")
    packed = torch.empty((R, emb.emb_row_bytes(D, "mxfp4")), dtype=torch.uint8, device=H.DEV)
    back = torch.empty((R, D), dtype=torch.bfloat16, device=H.DEV)
    _, off, rows = _batch(rng, 1, B, R, 12)
    rows_dev, off_dev = H.dev(rows), H.dev(off)
    hot = H.dev(np.arange(0, R, 3, dtype=np.int64))
    cache = torch.empty((hot.numel(), packed.shape[1]), dtype=torch.uint8, device=H.DEV)
    index = torch.empty(emb.emb_cache_index_bytes(R), dtype=torch.uint8, device=H.DEV)
    pooled, either = (torch.empty((1, B, D), device=H.DEV) for _ in range(2))
    scores = torch.empty((B, R), dtype=torch.bfloat16, device=H.DEV)
    few = torch.empty((1, R), device=H.DEV)
    st = _status()
    ts = emb.TableSet([packed], D, "mxfp4")

    def chain():
        emb.emb_quantize_rows_from(t, "mxfp4", packed)
        emb.emb_dequantize_rows(packed, "mxfp4", back)
        emb.emb_bag_forward(ts, rows_dev, off_dev, B, "sum", pooled, st)
        emb.emb_rows_product(pooled[0], packed, D, scores)
        emb.emb_rows_product(packed[:1], packed, D, few)
        emb.emb_cache_build_quantized(t.data_ptr(), R, D, "f32", "mxfp4", hot, cache, index, st)
        emb.emb_bag_forward_cached_quantized(t.data_ptr(), R, D, "f32", "mxfp4", cache, index, hot.numel(), rows_dev, off_dev, B,
                                             "sum", either, None, st)
        return [z.clone() for z in (packed, back, pooled, scores, few, cache, either)]

    chain()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream(device=H.DEV)
    with torch.cuda.graph(graph, stream=stream):
        chain()
    for k in range(4):
        t.copy_(_src(np.random.default_rng(50 + k), R, D, "f32")[0])
        rows_dev.copy_(H.dev(np.random.default_rng(60 + k).integers(0, R, size=rows.size).astype(np.int64)))
        want = chain()
        torch.cuda.synchronize()
        for z in (packed, back, pooled, scores, few, cache, either):
            z.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for z, w in zip((packed, back, pooled, scores, few, cache, either), want):
            assert torch.equal(z, w)
    assert st.item() == 0


def test_two_streams_at_once():
    rng = np.random.default_rng(43)
    D, N = 256, 5000
    w = mx.random_rows(rng, N, D, 118, 129)
    wd = H.dev(w)
    xs = [_operand(rng, 48, D, "bf16") for _ in range(2)]
    outs = [torch.empty((48, N), device=H.DEV) for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(device=H.DEV) for _ in range(2)]
    for _ in range(5):
        for (x, _), o, s in zip(xs, outs, streams):
            with torch.cuda.stream(s):
                emb.emb_rows_product(x, wd, D, o)
    torch.cuda.synchronize()
    for (_, xv), o in zip(xs, outs):
        _check_product(o.cpu().double().numpy(), xv, mx.values(w, D), "bf16", "f32")
