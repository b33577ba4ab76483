"""The 4-bit KV cache's writes and reads against the codec's definition (needs a B200 for the kernels)."""
import numpy as np
import pytest
import torch

import paper_2604_11035_b200 as isd_pkg
from paper_2604_11035_b200.binding import ST_BAD_PAGE_ID
from quant_ref import Cache, D, PAGE, TILE, encode, pack, random_cache, unpack

DEV = "cuda:0"


def make(heads, pages):
    return isd_pkg.Isd(batch=1, stride=1, n_q_heads=heads, n_kv_heads=heads, vocab=64, max_pages_per_slot=4,
                       num_pages=pages, logits_dtype="f32")


def hard_rows(heads, seed):
    """Rows where a 4-bit codec can go wrong, bf16 [n, heads, 128]."""
    rng = np.random.default_rng(seed)
    n = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    rows = [n(heads, D), np.zeros((heads, D)), np.full((heads, D), 2.5), np.full((heads, D), -0.75),  # one sign only
            np.abs(n(heads, D)) + 1, -np.abs(n(heads, D)) - 1,
            np.arange(D)[None].repeat(heads, 0) / 8.0,                       # quotients that are ties (s = 127/8/15 -> bf16)
            np.where(np.arange(D) % 2, 7.5, -7.5)[None].repeat(heads, 0),     # s = 1: ties and the ends of the range
            (rng.integers(-15, 16, (heads, D)) / 2.0).clip(-7.5, 7.5),
            n(heads, D) * 1e-38, n(heads, D) * 1e-40, n(heads, D) * 1e36, n(heads, D) * 3e-31, n(heads, D) * 2e30]
    one = n(heads, D)
    one[:, 5] = 300.0                                                        # an outlier
    rows.append(one)
    eps = np.full((heads, D), 1e-30)
    eps[:, 0] = 1.0
    rows.append(eps)
    for bad in (np.nan, np.inf, -np.inf):
        x = n(heads, D)
        x[:, 77] = bad
        rows.append(x)
    big = n(heads, D)
    big[:, 0], big[:, 1] = 3.0e38, -3.0e38                                   # the range overflows
    rows.append(big)
    return torch.from_numpy(np.stack(rows).astype(np.float32)).bfloat16()


def same_tiles(got, want):
    """Bitwise, but for the payload of a NaN scale."""
    gc, gs, gz = unpack(got)
    wc, ws, wz = unpack(want)
    for a, b in zip(gc, wc):
        assert np.array_equal(a, b)
    for a, b in zip((*gs, *gz), (*ws, *wz)):
        assert np.array_equal(a, b, equal_nan=True)


def test_reference_codec_by_hand():
    c, s, z = encode(np.array([-7.5, 7.5, 0.5, 1.5, -0.5] + [0.0] * 123))
    assert s == 1.0 and z == 8  # round(7.5) = 8, the even side
    assert c[:5].tolist() == [0, 15, 8, 10, 8]  # -8 + 8; 8 + 8 cut to 15; ties 0.5 -> 0, 1.5 -> 2, -0.5 -> 0
    cache = random_cache(3, 2, 1)
    codes, scales, zeros = unpack(pack(cache))
    for i in range(2):
        assert np.array_equal(codes[i], cache.c[i]) and np.array_equal(scales[i], cache.s[i]) and np.array_equal(zeros[i], cache.z128[i])


def test_entry_points_refuse_a_missing_context():
    lib = isd_pkg.load()
    for name in ("isd_kv_write_quant", "isd_kv_read_quant", "isd_logprobs"):
        assert getattr(lib, name)(None, None, None) == -1
    assert lib.isd_admit(None, None, None, None) == -1
    assert lib.isd_attn_quant(None, None, None, None, None, None, None, None, None) == -1
    assert lib.isd_step_quant(None, None, None, 1, None, None, None, 0, None) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [1, 2, 5, 8])
@pytest.mark.parametrize("order", ["runs", "shuffled"])
def test_write_matches_the_definition_and_leaves_the_rest(heads, order):
    rows = torch.cat([hard_rows(heads, 3), torch.randn(75, heads, D, generator=torch.Generator().manual_seed(5)).bfloat16()])
    T, pages = rows.shape[0], 17
    rng = np.random.default_rng(heads)
    if order == "runs":  # three requests, each from a page's start or from its middle, with padding between them
        slot = np.concatenate([np.arange(3 * 16, 3 * 16 + 37), [-1, -7], np.arange(9 * 16 + 5, 9 * 16 + 30),
                               np.arange(0, T - 37 - 2 - 25) + 12 * 16])[:T]
    else:
        slot = rng.permutation(pages * PAGE)[:T]
        slot[rng.integers(0, T, 5)] = -3
    start = random_cache(pages, heads, 11)
    pool = torch.from_numpy(pack(start)).to(DEV)
    k, v = rows.to(DEV), rows.flip(0).contiguous().to(DEV)
    make(heads, pages).isd_kv_write_quant(k, v, torch.from_numpy(slot).to(DEV), pool)
    kn, vn = k.cpu().float().numpy(), v.cpu().float().numpy()
    for t, s in enumerate(slot):
        if s >= 0:
            start.store(s // PAGE, s % PAGE, kn[t], vn[t])
    same_tiles(pool.cpu().numpy(), pack(start))


@pytest.mark.gpu
@pytest.mark.parametrize("T", [0, 1, 15, 16, 17, 33])
def test_write_then_read_strided_rows(T):
    heads, pages = 3, 6
    g = torch.Generator().manual_seed(T)
    fused = torch.randn(T, 4 * heads, D, generator=g).bfloat16().to(DEV)
    k, v = fused[:, heads:2 * heads], fused[:, 3 * heads:]
    slot = torch.arange(T, dtype=torch.int64, device=DEV) + 21
    isd = make(heads, pages)
    pool = isd_pkg.alloc_kv_pool_quant(pages, heads, DEV)
    isd.isd_kv_write_quant(k, v, slot, pool)
    room = torch.full((T, 4 * heads, D), 7.0, dtype=torch.bfloat16, device=DEV)
    if T > 2:
        slot = slot.clone()
        slot[1] = -1
    isd.isd_kv_read_quant(pool, slot, room[:, :heads], room[:, 2 * heads:3 * heads])
    for x, back in ((k, room[:, :heads]), (v, room[:, 2 * heads:3 * heads])):
        c, s, z = encode(x.cpu().float().numpy()) if T else (np.zeros((0, heads, D)), np.zeros((0, heads)), np.zeros((0, heads)))
        want = torch.from_numpy((s[..., None] * (c.astype(np.float64) - z[..., None])).astype(np.float32)).bfloat16()
        if T > 2:
            want[1] = 7.0
        assert torch.equal(back.cpu(), want)
    assert bool((room[:, heads:2 * heads] == 7).all()) and bool((room[:, 3 * heads:] == 7).all())


@pytest.mark.gpu
def test_read_of_hard_rows_and_any_order():
    heads, pages = 2, 8
    rows = hard_rows(heads, 9)
    T = rows.shape[0]
    slot = torch.from_numpy(np.random.default_rng(2).permutation(pages * PAGE)[:T]).to(DEV)
    isd, pool = make(heads, pages), isd_pkg.alloc_kv_pool_quant(pages, heads, DEV)
    isd.isd_kv_write_quant(rows.to(DEV), rows.to(DEV), slot, pool)
    k, v = (torch.zeros(T, heads, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    isd.isd_kv_read_quant(pool, slot, k, v)
    c, s, z = encode(rows.float().numpy())
    with np.errstate(all="ignore"):
        want = torch.from_numpy((s[..., None] * (c.astype(np.float64) - z[..., None])).astype(np.float32)).bfloat16()
    for got in (k, v):
        assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(want))


@pytest.mark.gpu
def test_slots_behind_the_pool_are_reported_and_skipped():
    heads, pages = 2, 4
    isd, pool = make(heads, pages), isd_pkg.alloc_kv_pool_quant(pages, heads, DEV)
    before = pool.clone()
    rows = torch.randn(3, heads, D, device=DEV).bfloat16()
    isd.isd_kv_write_quant(rows, rows, torch.tensor([pages * PAGE, 1 << 40, -1], device=DEV), pool)
    assert isd.isd_read_status() == ST_BAD_PAGE_ID and torch.equal(pool, before)
    k = torch.full((3, heads, D), 3.0, dtype=torch.bfloat16, device=DEV)
    isd.isd_kv_read_quant(pool, torch.tensor([pages * PAGE, 0, -1], device=DEV), k, k.clone())
    assert isd.isd_read_status() == ST_BAD_PAGE_ID
    assert bool((k[0] == 3).all()) and bool((k[1] == 0).all()) and bool((k[2] == 3).all())


@pytest.mark.gpu
def test_refusals():
    heads, pages = 2, 4
    isd, pool = make(heads, pages), isd_pkg.alloc_kv_pool_quant(pages, heads, DEV)
    rows, slot = torch.zeros(3, heads, D, dtype=torch.bfloat16, device=DEV), torch.arange(3, device=DEV)
    isd.isd_kv_write_quant(rows, rows, slot, pool)
    for k, s, p in ((rows.float(), slot, pool), (rows[:2], slot, pool), (rows, slot.int(), pool), (rows, slot, pool[:3]),
                    (rows, slot.cpu(), pool), (rows.cpu(), slot, pool), (rows.transpose(1, 2).contiguous().transpose(1, 2), slot, pool),
                    (torch.zeros(3, heads * D + 4, dtype=torch.bfloat16, device=DEV)[:, :heads * D].view(3, heads, D), slot, pool)):
        with pytest.raises(isd_pkg.IsdError):
            isd.isd_kv_write_quant(k, rows, s, p)
    odd = torch.zeros(3 * heads * D + 8, dtype=torch.bfloat16, device=DEV)[1:1 + 3 * heads * D].view(3, heads, D)
    with pytest.raises(isd_pkg.IsdError, match="aligned"):
        isd.isd_kv_write_quant(odd, rows, slot, pool)


@pytest.mark.gpu
def test_pool_behind_four_gigabytes():
    heads = 8
    pages = (1 << 32) // (heads * TILE) + 40  # the last pages start behind byte 2^32
    isd = make(heads, pages)
    pool = torch.empty(pages, heads, TILE, dtype=torch.uint8, device=DEV)
    T = 40
    rows = torch.randn(T, heads, D, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    slot = torch.arange(T, device=DEV) + (pages - 3) * PAGE
    isd.isd_kv_write_quant(rows, rows, slot, pool)
    k, v = torch.zeros_like(rows), torch.zeros_like(rows)
    isd.isd_kv_read_quant(pool, slot, k, v)
    c, s, z = encode(rows.cpu().float().numpy())
    want = torch.from_numpy((s[..., None] * (c.astype(np.float64) - z[..., None])).astype(np.float32)).bfloat16()
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), want)
