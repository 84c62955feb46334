"""GPU parity of the operations on a KV cache held in 8 or 4 bits, against the fp64 oracle.

Codes and scales are defined to the bit, so writing and reading back are compared exactly; the attention
tolerances are derived in quant_utils.check_out.
"""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2606_00144_amd as bd
from gpu_utils import bf16_dev, bf16_host64, case, i32_dev, poison_workspace
from quant_utils import (check_out, garbage, make_cache, rows, special_rows, to_dev, to_host, to_pages,
                         values_as_bits)

pytestmark = pytest.mark.gpu
BITS = pytest.mark.parametrize("bits", [4, 8])


def _u16(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


# ------------------------------------------------------------------ writing and reading back

@BITS
@pytest.mark.parametrize("n", [1, 6, 16, 17, 150])
def test_append_writes_the_defined_bytes(bits, n):
    # up to 16 rows one launch advances the lengths too; all other bytes stay as they are
    S, Hkv, cap = 3, 5, 160
    lens = [0, 7, 160 - n // 2 - 1]
    cache = tuple(garbage((S, Hkv, cap, w), 3 + w) for w in (16 * bits, 16 * bits, 4, 4))
    kn = special_rows(S * n * Hkv, 5).reshape(S, n, Hkv, 128)
    vn = special_rows(S * n * Hkv, 6).reshape(S, n, Hkv, 128)
    want, ol = O.cache_append_q(cache, lens, kn, vn, bits)
    case(f"append_q bits={bits} n={n}")
    dev, ld = to_dev(cache), i32_dev(lens)
    bd.bd_cache_append_q(dev, ld, bf16_dev(kn), bf16_dev(vn))
    torch.cuda.synchronize()
    assert ld.cpu().tolist() == ol.tolist()
    for name, a, b in zip(bd.QuantKV._fields, to_host(dev), want):
        assert np.array_equal(a, b), (name, np.argwhere(a != b)[:5])


@BITS
@pytest.mark.parametrize("n", [5, 40])
def test_append_counts_lists_and_capacity(bits, n):
    S, Hkv, cap, ld = 5, 2, 100, 30
    lens, counts, nsel = [10, 95, 100, 0, 50], [n, n - 1, 3, 0, -4], [5, 25, 30, 0, 9]
    cache = tuple(garbage((S, Hkv, cap, w), w) for w in (16 * bits, 16 * bits, 4, 4))
    idx = np.full((S, Hkv, ld), -1, np.int32)
    kn, vn = rows((S, n, Hkv, 128), 1), rows((S, n, Hkv, 128), 2)
    want, ol, oi, on = O.cache_append_q(cache, lens, kn, vn, bits, counts, idx, nsel)
    case(f"append_q counts bits={bits} n={n}")
    dev, l, i, m = to_dev(cache), i32_dev(lens), i32_dev(idx), i32_dev(nsel)
    bd.bd_cache_append_q(dev, l, bf16_dev(kn), bf16_dev(vn), counts=i32_dev(counts), idx=i, nsel=m)
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(to_host(dev), want))
    assert l.cpu().tolist() == ol.tolist() and m.cpu().tolist() == on.tolist()
    assert np.array_equal(i.cpu().numpy(), oi)


@BITS
@pytest.mark.parametrize("page,n", [(16, 6), (24, 40), (1, 5), (64, 20)])
def test_append_and_read_paged(bits, page, n):
    S, Hkv, cap = 3, 2, 192
    lens = [30, 0, 100]
    cache, _, _ = make_cache(S, Hkv, cap, bits, lens, 40)
    kn, vn = rows((S, n, Hkv, 128), 41), rows((S, n, Hkv, 128), 42)
    want, ol = O.cache_append_q(cache, lens, kn, vn, bits)
    pool, table = to_pages(cache, [L + n for L in lens], page, 43)
    case(f"append_q paged bits={bits} page={page} n={n}")
    dev, l, td = to_dev(pool), i32_dev(lens), i32_dev(table)
    bd.bd_cache_append_q(dev, l, bf16_dev(kn), bf16_dev(vn), page_table=td)
    k, v = bd.bd_cache_read_q(dev, l, 150, page_table=td)
    torch.cuda.synchronize()
    assert l.cpu().tolist() == ol.tolist()
    for got, c, s in ((k, 0, 2), (v, 1, 3)):
        for i, L in enumerate(ol):
            m = min(int(L), 150)
            assert np.array_equal(_u16(got[i, :, :m]), values_as_bits(want[c][i, :, :m], want[s][i, :, :m], bits))
            assert not _u16(got[i, :, m:]).any()
    # pages that no new row touches keep their bytes
    used = {int(table[s, t // page]) for s in range(S) for t in range(lens[s], lens[s] + n)}
    for a, b in zip(to_host(dev), pool):
        keep = [p for p in range(b.shape[0]) if p not in used]
        assert np.array_equal(a[keep], b[keep])


@BITS
def test_rows_of_pages_outside_the_pool(bits):
    # dropped when written, zero when read
    Hkv, page = 2, 16
    lens = [40]
    cache, kb, _ = make_cache(1, Hkv, 64, bits, lens, 50)
    pool, table = to_pages(cache, [64], page, 51)
    bad = table.copy()
    bad[0, 1], bad[0, 2] = -1, pool[0].shape[0]
    case(f"out-of-pool pages bits={bits}")
    dev, l, td = to_dev(pool), i32_dev(lens), i32_dev(bad)
    k, _ = bd.bd_cache_read_q(dev, l, 48, page_table=td, with_v=False)
    kn = rows((1, 20, Hkv, 128), 52)
    bd.bd_cache_append_q(dev, l, bf16_dev(kn), bf16_dev(kn), page_table=td)
    torch.cuda.synchronize()
    assert np.array_equal(_u16(k[0, :, :16]), kb[0, :, :16]) and not _u16(k[0, :, 16:]).any()
    assert l.cpu().tolist() == [60]
    c, s = O.mx_quantise(kn[0, 8:20].transpose(1, 0, 2), bits)       # positions 48 .. 59, in the pool
    host = to_host(dev)
    assert np.array_equal(host[0][table[0, 3], :, :12], c) and np.array_equal(host[2][table[0, 3], :, :12], s)
    for pg in range(pool[0].shape[0]):
        if pg != table[0, 3]:
            assert all(np.array_equal(a[pg], b[pg]) for a, b in zip(host, pool)), pg


@BITS
def test_read_first_and_strided_outputs(bits):
    S, Hkv, cap, n = 4, 3, 90, 30
    lens, first = [90, 20, 5, 0], [61, -3, 5, 0]
    cache, kb, vb = make_cache(S, Hkv, cap, bits, lens, 60)
    big = torch.full((2, S, n + 7, Hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda")   # token-major, rows to spare
    ko, vo = (big[i].transpose(1, 2)[:, :, 2:2 + n] for i in range(2))
    case(f"read_q strided bits={bits}")
    k, v = bd.bd_cache_read_q(to_dev(cache), i32_dev(lens), n, first=i32_dev(first), outputs=(ko, vo))
    torch.cuda.synchronize()
    assert k.data_ptr() == ko.data_ptr() and v.data_ptr() == vo.data_ptr()
    for got, ref in ((k, kb), (v, vb)):
        want = np.zeros((S, Hkv, n, 128), np.uint16)
        for s in range(S):
            for i in range(n):
                t = first[s] + i
                if 0 <= t < lens[s]:
                    want[s, :, i] = ref[s, :, t]
        assert np.array_equal(_u16(got.contiguous()), want)
    rest = torch.cat([big[:, :, :2], big[:, :, 2 + n:]], dim=2)
    assert bool((rest == 7.0).all())


@BITS
def test_special_values_read_back(bits):
    n = 400
    x = special_rows(n, 9).reshape(1, n, 1, 128)
    cache = bd.quant_kv_empty(1, 1, n, bits)
    l = i32_dev([0])
    case(f"special values bits={bits}")
    bd.bd_cache_append_q(cache, l, bf16_dev(x), bf16_dev(x[:, ::-1]))
    k, v = bd.bd_cache_read_q(cache, l, n)
    torch.cuda.synchronize()
    want = O.mx_values(*O.mx_quantise(x[0, :, 0], bits), bits)
    np.testing.assert_array_equal(bf16_host64(k)[0, 0], want)
    np.testing.assert_array_equal(bf16_host64(v)[0, 0], want[::-1])
    # every finite element of an ordinary block is within half a step of the top binade: 1 of 4..7, 16 of 256..464
    f = O.bf16_to_f64(x[0, :, 0]).reshape(n, 4, 32)
    a = np.abs(f).max(-1)
    with np.errstate(invalid="ignore"):
        ok = np.isfinite(a) & (a > 1e-30) & (a < 1e38)
        off = np.abs(want.reshape(n, 4, 32) - f).max(-1)
    assert (off[ok] <= a[ok] / (4 if bits == 4 else 16)).all()


# ------------------------------------------------------------------ verify

def _verify(S, Hq, Hkv, cap, lens, gamma, bits, seed, what, page=0, token_major=False, qs=1.0, **kw):
    cache, kb, vb = make_cache(S, Hkv, cap, bits, lens, seed)
    q = rows((S, gamma + 1, Hq, 128), seed + 5, qs)
    table = None
    if page:
        pool, table = to_pages(cache, lens, page, seed + 6)
        dev, table = to_dev(pool), i32_dev(table)
    elif token_major:                                        # rows of a position side by side: [S][L][Hkv]
        dev = bd.QuantKV(*[b.transpose(1, 2).contiguous().transpose(1, 2) for b in to_dev(cache)])
    else:
        dev = to_dev(cache)
    nb = bd.lib().bd_verify_attn_q_workspace_bytes(S, Hkv, Hq, gamma, cap)
    case(f"verify_q {what} bits={bits} S={S} heads={Hq}/{Hkv} lens={list(lens)[:6]} gamma={gamma} page={page}")
    out, lse = bd.bd_verify_attn_q(dev, bf16_dev(q), i32_dev(lens), return_lse=True, page_table=table, max_seq_len=cap,
                                   workspace=poison_workspace(nb), **kw)
    torch.cuda.synchronize()
    ref = lambda q, k, v: O.verify_attn(k, v, q, lens, gamma)
    ro, rl = ref(q, kb, vb)
    check_out(out, lse, ro, rl, kb, vb, q, ref, max(lens), what)
    return dev, q, out


@BITS
@pytest.mark.parametrize("L", [0, 1, 2, 5, 31, 32, 33, 127, 128, 129, 500, 2049])
def test_verify_lengths(bits, L):
    _verify(2, 8, 2, max(L, 1), [L, L], 5, bits, L, "length")


@BITS
@pytest.mark.parametrize("Hq,Hkv,gamma", [(4, 4, 0), (4, 4, 5), (8, 1, 0), (8, 2, 3), (40, 8, 2), (8, 1, 5), (16, 1, 8), (6, 2, 40)])
def test_verify_heads_and_rows(bits, Hq, Hkv, gamma):
    # 1 to 144 rows a KV head: one or two row tiles, several row blocks
    _verify(2, Hq, Hkv, 700, [700, 333], gamma, bits, Hq + gamma, "heads")


@BITS
@pytest.mark.parametrize("page", [16, 48, 64, 24, 1, 7])
def test_verify_paged(bits, page):
    _verify(5, 8, 2, 1500, [1500, 0, 1, 17, 700], 5, bits, page, "paged", page=page)


@BITS
def test_verify_token_major_and_capacity(bits):
    # a capacity far beyond the lengths: the split follows the lengths
    _verify(3, 8, 2, 6000, [40, 1, 129], 4, bits, 77, "capacity", token_major=True)


@BITS
@pytest.mark.parametrize("S", [64, 65, 200])
def test_verify_many_sequences(bits, S):
    r = np.random.default_rng(S)
    lens = r.integers(0, 90, S).tolist()
    lens[3], lens[-1] = 400, 257
    _verify(S, 4, 2, 400, lens, 2, bits, S, "many sequences")


@BITS
@pytest.mark.parametrize("page", [0, 16, 24])
@pytest.mark.parametrize("Hq,Hkv,gamma", [(8, 1, 4), (8, 2, 8), (16, 2, 8)])
def test_verify_more_than_32_rows(bits, page, Hq, Hkv, gamma):
    # 40, 36 and 72 rows a KV head, in a capacity that calls for blocks of three row tiles (24-row pages: of two)
    S, have, cap = 6, 5000, 65536
    lens = [have, 33, 0, 1200, 700, 64]
    cache, kb, vb = make_cache(S, Hkv, have, bits, lens, Hq + gamma)
    q = rows((S, gamma + 1, Hq, 128), Hq + gamma + 5)
    table = None
    if page:
        pool, table = to_pages(cache, lens, page, 6)
        cap = cap // page * page
        wide = np.full((S, cap // page), -1, np.int32)
        wide[:, :table.shape[1]] = table
        dev, table = to_dev(pool), i32_dev(wide)
    else:
        dev = bd.quant_kv_empty(S, Hkv, cap, bits)
        for b, h in zip(dev, to_dev(cache)):
            b.fill_(255)
            b[:, :, :have] = h
    case(f"verify_q many rows bits={bits} heads={Hq}/{Hkv} gamma={gamma} page={page}")
    nb = bd.lib().bd_verify_attn_q_workspace_bytes(S, Hkv, Hq, gamma, cap)
    out, lse = bd.bd_verify_attn_q(dev, bf16_dev(q), i32_dev(lens), return_lse=True, page_table=table, max_seq_len=cap,
                                   workspace=poison_workspace(nb))
    torch.cuda.synchronize()
    ref = lambda q, k, v: O.verify_attn(k, v, q, lens, gamma)
    check_out(out, lse, *ref(q, kb, vb), kb, vb, q, ref, have, "many rows")


@BITS
@pytest.mark.parametrize("S,Hkv,top", [(24, 4, 2600), (9, 8, 900), (60, 2, 700), (3, 2, 5000), (40, 4, 300)])
def test_verify_ragged_batches(bits, S, Hkv, top):
    # units with shares of their own of every length, shares of two units, short units that are not cut
    r = np.random.default_rng(S + bits)
    lens = np.exp(r.uniform(np.log(20), np.log(top), S)).astype(int).tolist()
    lens[0], lens[1] = top, 0
    _verify(S, 2 * Hkv, Hkv, top, lens, 4, bits, S, "ragged", page=16 if S % 2 else 0)


@pytest.mark.parametrize("bits,L,Hkv,page", [(4, 20000, 1, 0), (8, 20000, 1, 16), (4, 9000, 3, 0), (4, 70000, 1, 16), (8, 5000, 1, 24)])
def test_verify_one_long_sequence(bits, L, Hkv, page):
    # units of many pieces: the two-level merge; tables filled more than once
    _verify(1, 4 * Hkv, Hkv, L, [L], 5, bits, 90, "long", page=page)


def test_verify_large_scores():
    # weights concentrate on few keys, maxima rise tile by tile
    _verify(2, 8, 2, 900, [900, 850], 5, 4, 91, "large scores", qs=20.0)


@BITS
@pytest.mark.parametrize("page", [0, 16, 24])
def test_values_past_the_rows_that_see_them_do_not_matter(bits, page):
    # a draft's key and value that are not numbers reach the rows from its position on, in the blocks they stand in
    S, Hq, Hkv, gamma, cap = 1, 4, 2, 5, 90
    lens = [87]
    cache, kb, vb = make_cache(S, Hkv, cap, bits, lens, 95)
    q = rows((S, gamma + 1, Hq, 128), 96)
    ro, _ = O.verify_attn(kb, vb, q, lens, gamma)
    cache[3][0, 0, 84, 1] = 255            # V of position 84 (row 3), head 0, elements 32 .. 63
    cache[2][0, 1, 85, 2] = 255            # K of position 85 (row 4), head 1
    table = None
    dev = cache
    if page:
        dev, table = to_pages(cache, lens, page, 97)
        table = i32_dev(table)
    case(f"NaN in later drafts bits={bits} page={page}")
    out = bd.bd_verify_attn_q(to_dev(dev), bf16_dev(q), i32_dev(lens), page_table=table, max_seq_len=cap)
    torch.cuda.synchronize()
    got = bf16_host64(out)
    nan = np.zeros(got.shape, bool)
    nan[0, 3:, :2, 32:64] = True
    nan[0, 4:, 2:] = True
    assert np.array_equal(np.isnan(got), nan)
    np.testing.assert_allclose(got[~nan], ro[~nan], rtol=2e-2, atol=2e-2)


@BITS
@pytest.mark.parametrize("page", [16, 24])
def test_verify_pages_outside_the_pool(bits, page):
    # their keys are absent: the result is that of a sequence without them
    S, Hq, Hkv, L, gamma = 1, 4, 2, 200, 3
    cache, kb, vb = make_cache(S, Hkv, L, bits, [L], 98)
    pool, table = to_pages(cache, [L], page, 99)
    table[0, 1], table[0, 4] = -7, pool[0].shape[0] + 5
    gone = np.r_[page:2 * page, 4 * page:5 * page]
    keep = np.setdiff1d(np.arange(L), gone)
    q = rows((S, gamma + 1, Hq, 128), 100)
    case(f"verify out-of-pool pages bits={bits} page={page}")
    out, lse = bd.bd_verify_attn_q(to_dev(pool), bf16_dev(q), i32_dev([L]), page_table=i32_dev(table), max_seq_len=L,
                                   return_lse=True)
    torch.cuda.synchronize()
    ref = lambda q, k, v: O.verify_attn(k[:, :, keep], v[:, :, keep], q, [keep.size], gamma)
    check_out(out, lse, *ref(q, kb, vb), kb, vb, q, ref, L, "out of pool")


def test_nan_queries_and_infinite_scores():
    cache, kb, vb = make_cache(1, 1, 70, 4, [70], 101)
    q = rows((1, 3, 2, 128), 102)
    q[0, 1, 0, 7] = 0x7FC0
    case("NaN query")
    out, lse = bd.bd_verify_attn_q(to_dev(cache), bf16_dev(q), i32_dev([70]), return_lse=True)
    torch.cuda.synchronize()
    got, gl = bf16_host64(out), lse.cpu().numpy()
    bad = np.zeros((1, 3, 2), bool)
    bad[0, 1, 0] = True
    assert np.isnan(got[bad]).all() and np.isnan(gl[bad]).all()
    assert not np.isnan(got[~bad]).any() and not np.isnan(gl[~bad]).any()


def test_rows_beyond_32_bits_of_bytes():
    # row numbers whose byte offsets pass 2^32, in both layouts
    bits, Hkv, far = 4, 1, (1 << 26) + 12345                 # 64-byte rows: 4.3 GB apart
    L, gamma = 300, 2
    cache, kb, vb = make_cache(2, Hkv, L, bits, [L, L], 103)
    q = rows((2, gamma + 1, 4, 128), 104)
    ref = lambda q, k, v: O.verify_attn(k, v, q, [L, L], gamma)
    ro, rl = ref(q, kb, vb)
    big = [torch.empty((far + 1000) * w, dtype=torch.uint8, device="cuda") for w in (64, 64, 4, 4)]
    dev = bd.QuantKV(*[b.as_strided((2, Hkv, L, w), (far * w, 0, w, 1)) for b, w in zip(big, (64, 64, 4, 4))])
    for d, h in zip(dev, to_dev(cache)):
        d.copy_(h)
    case("byte offsets past 2^32, contiguous")
    out, lse = bd.bd_verify_attn_q(dev, bf16_dev(q), i32_dev([L, L]), return_lse=True)
    torch.cuda.synchronize()
    check_out(out, lse, ro, rl, kb, vb, q, ref, L, "far rows")
    n_new = 3
    kn = rows((2, n_new, Hkv, 128), 105)
    l = i32_dev([L - n_new, L - n_new])
    bd.bd_cache_append_q(dev, l, bf16_dev(kn), bf16_dev(kn))
    k, v = bd.bd_cache_read_q(dev, l, n_new, first=i32_dev([L - n_new] * 2))
    torch.cuda.synchronize()
    want = values_as_bits(*O.mx_quantise(kn.transpose(0, 2, 1, 3), bits), bits)
    assert np.array_equal(_u16(k), want) and np.array_equal(_u16(v), want)


# ------------------------------------------------------------------ sparse decode

def _decode(cache, kb, vb, q, idx, nsel, lens, what, table=None, cap=None):
    case(f"decode_q {what}")
    S, Hq = q.shape[:2]
    nb = bd.lib().bd_sparse_decode_attn_q_workspace_bytes(S, kb.shape[1], Hq, idx.shape[2])
    out, lse = bd.bd_sparse_decode_attn_q(to_dev(cache), bf16_dev(q), i32_dev(idx), i32_dev(nsel), i32_dev(lens),
                                          return_lse=True, page_table=table, max_seq_len=cap, workspace=poison_workspace(nb))
    torch.cuda.synchronize()
    clip = np.clip(np.asarray(nsel), 0, idx.shape[2])
    ref = lambda q, k, v: O.sparse_decode_attn(k, v, q, idx, clip, lens)
    check_out(out, lse, *ref(q, kb, vb), kb, vb, q, ref, max(1, idx.shape[2]), what)


@BITS
@pytest.mark.parametrize("B", [1, 31, 33, 256, 1000])
@pytest.mark.parametrize("page", [0, 16, 24])
def test_decode_lists(bits, B, page):
    S, Hq, Hkv, cap = 3, 8, 2, 1300
    lens = [1300, 40, 700]
    cache, kb, vb = make_cache(S, Hkv, cap, bits, lens, 110)
    g = np.random.default_rng(B)
    idx = np.full((S, Hkv, B), -1, np.int32)
    for s in range(S):
        for h in range(Hkv):
            m = min(B, lens[s])
            idx[s, h, :m] = g.permutation(lens[s])[:m]          # any order
    q = rows((S, Hq, 128), 111)
    table = None
    if page:
        cache, table = to_pages(cache, lens, page, 112)
        table = i32_dev(table)
    _decode(cache, kb, vb, q, idx, [min(B, L) for L in lens], lens, f"bits={bits} B={B} page={page}", table, cap)


@BITS
def test_decode_odd_entries(bits):
    # absent entries, entries past the length, duplicates, counts outside the list, no entries at all
    S, Hq, Hkv, cap, ld = 6, 6, 2, 200, 70
    lens = [200, 100, 3, 0, 150, 60]
    cache, kb, vb = make_cache(S, Hkv, cap, bits, lens, 120)
    g = np.random.default_rng(7)
    idx = g.integers(-40, 260, (S, Hkv, ld)).astype(np.int32)
    idx[4] = 17                                                 # one position ld times
    idx[5, 0], idx[5, 1] = -1, 99                               # a list of nothing visible
    nsel = [ld, 1000, 5, ld, ld, 66]
    q = rows((S, Hq, 128), 121)
    _decode(cache, kb, vb, q, idx, nsel, lens, f"odd entries bits={bits}")
    _decode(cache, kb, vb, q, idx, [0, -5, 1, 0, 2, 0], lens, f"short counts bits={bits}")
    _decode(cache, kb, vb, q, np.zeros((S, Hkv, 0), np.int32), [0] * S, lens, f"empty list bits={bits}")


@BITS
def test_decode_long_list_of_few_heads(bits):
    # a list longer than the table, split over many workgroups; then many whole lists per workgroup
    cache, kb, vb = make_cache(1, 1, 9000, bits, [9000], 130)
    g = np.random.default_rng(8)
    idx = g.permutation(9000).astype(np.int32)[None, None]
    _decode(cache, kb, vb, rows((1, 16, 128), 131), idx, [9000], [9000], f"long list bits={bits}")
    S, Hkv = 40, 16
    lens = g.integers(0, 120, S).tolist()
    cache, kb, vb = make_cache(S, Hkv, 120, bits, lens, 132)
    idx = g.integers(0, 120, (S, Hkv, 90)).astype(np.int32)
    _decode(cache, kb, vb, rows((S, 32, 128), 133), idx, [90] * S, lens, f"many lists bits={bits}")


# ------------------------------------------------------------------ as a program uses them

def test_results_do_not_depend_on_the_run():
    cache, kb, vb = make_cache(3, 2, 4000, 4, [4000, 1, 2500], 140)
    dev, q, l = to_dev(cache), bf16_dev(rows((3, 6, 8, 128), 141)), i32_dev([4000, 1, 2500])
    case("verify_q repeated")
    ws = bd.Workspace()
    first = bd.bd_verify_attn_q(dev, q, l, workspace=ws)
    for _ in range(5):
        again = bd.bd_verify_attn_q(dev, q, l, workspace=ws)
        assert torch.equal(again.view(torch.int16), first.view(torch.int16))
    assert not ws.buf[(-ws.buf.data_ptr()) % 256:][:1 << 20].any()      # counters are zero again


def test_workspace_between_operations_and_shapes():
    # one workspace for every call of a stream, quantised and bf16 alike
    cache, kb, vb = make_cache(2, 2, 3000, 8, [3000, 900], 150)
    dev, l = to_dev(cache), i32_dev([3000, 900])
    k16, v16 = bd.bd_cache_read_q(dev, l, 3000)
    q = rows((2, 6, 8, 128), 151)
    idx = np.stack([np.sort(np.random.default_rng(s).permutation(900)[:300]) for s in range(4)]).reshape(2, 2, 300).astype(np.int32)
    ws = bd.Workspace()
    case("one workspace for all")
    for _ in range(2):
        a = bd.bd_verify_attn_q(dev, bf16_dev(q), l, workspace=ws)
        b = bd.bd_verify_attn(k16, v16, bf16_dev(q), l, workspace=ws)
        c = bd.bd_sparse_decode_attn_q(dev, bf16_dev(q[:, 0]), i32_dev(idx), i32_dev([300, 300]), l, workspace=ws)
        d = bd.bd_sparse_decode_attn(k16, v16, bf16_dev(q[:, 0]), i32_dev(idx), i32_dev([300, 300]), l, workspace=ws)
        torch.cuda.synchronize()
        # the same values through the bf16 operations: both round their weights, and their outputs, to bf16
        np.testing.assert_allclose(bf16_host64(a), bf16_host64(b), atol=2e-2, rtol=1e-2)
        np.testing.assert_allclose(bf16_host64(c), bf16_host64(d), atol=2e-2, rtol=1e-2)


def test_graphs_replayed_side_by_side():
    # two graphs captured on one stream without a workspace do not share scratch, and follow the lengths
    cache, kb, vb = make_cache(2, 2, 5000, 4, [5000, 3000], 160)
    dev, q = to_dev(cache), bf16_dev(rows((2, 6, 8, 128), 161))
    lens = [i32_dev([5000, 3000]), i32_dev([700, 31])]
    outs = [torch.empty_like(q) for _ in lens]
    case("graphs")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for l, o in zip(lens, outs):
            bd.bd_verify_attn_q(dev, q, l, out=o)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for l, o in zip(lens, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            bd.bd_verify_attn_q(dev, q, l, out=o)
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for r in range(4):
        new = [[5000 - 700 * r, 3000 - r], [700 + 900 * r, 31 + r]]
        for l, n in zip(lens, new):
            l.copy_(i32_dev(n))
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for n, o in zip(new, outs):
            want = bd.bd_verify_attn_q(dev, q, i32_dev(n))
            torch.cuda.synchronize()
            assert torch.equal(o.view(torch.int16), want.view(torch.int16)), r


@BITS
def test_sequences_that_share_pages(bits):
    # a common prefix kept once: every sequence's table begins with the same pages
    S, Hq, Hkv, L, gamma, page = 4, 8, 2, 320, 3, 16
    lens = [320, 257, 300, 100]
    cache, kb, vb = make_cache(1, Hkv, L, bits, [L], 180)
    pool, table = to_pages(cache, [L], page, 181)
    kb, vb = np.repeat(kb, S, 0), np.repeat(vb, S, 0)
    q = rows((S, gamma + 1, Hq, 128), 182)
    kw = dict(page_table=i32_dev(np.repeat(table, S, 0)), max_seq_len=L)
    case(f"shared pages bits={bits}")
    dev = to_dev(pool)
    out, lse = bd.bd_verify_attn_q(dev, bf16_dev(q), i32_dev(lens), return_lse=True, **kw)
    k, v = bd.bd_cache_read_q(dev, i32_dev(lens), L, **kw)
    torch.cuda.synchronize()
    ref = lambda q, k, v: O.verify_attn(k, v, q, lens, gamma)
    check_out(out, lse, *ref(q, kb, vb), kb, vb, q, ref, L, "shared pages")
    for s, n in enumerate(lens):
        assert np.array_equal(_u16(k)[s, :, :n], kb[s, :, :n]) and np.array_equal(_u16(v)[s, :, :n], vb[s, :, :n])
        assert not _u16(k)[s, :, n:].any() and not _u16(v)[s, :, n:].any()


def test_calls_on_two_streams():
    # default scratch is a stream's own: calls that overlap give what they give alone
    S, L = 2, 9000
    cache, kb, vb = make_cache(S, 2, L, 4, [L, L], 190)
    dev, lens = to_dev(cache), [i32_dev([9000, 4000]), i32_dev([33, 8000])]
    qs = [bf16_dev(rows((S, 6, 8, 128), 191 + i)) for i in range(2)]
    idx = i32_dev(np.random.default_rng(3).integers(0, L, (S, 2, 700)).astype(np.int32))
    nsel = i32_dev([700, 650])
    both = lambda i: (bd.bd_verify_attn_q(dev, qs[i], lens[i]),
                      bd.bd_sparse_decode_attn_q(dev, qs[i][:, 0].contiguous(), idx, nsel, lens[i]))
    case("two streams")
    want = [both(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [[], []]
        for _ in range(4):
            for i, st in enumerate(streams):
                with torch.cuda.stream(st):
                    got[i].append(both(i))
        torch.cuda.synchronize()
        for i in range(2):
            for a in got[i]:
                assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(a, want[i]))


@BITS
def test_a_round_captured_and_replayed(bits):
    # append, draft, verification and rollback in one graph; each replay grows the caches as the eager round does
    S, Hq, Hkv, cap, L0, gamma = 2, 8, 2, 600, [130, 401], 3
    cache, kb, vb = make_cache(S, Hkv, cap, bits, L0, 200)
    kn, vn = bf16_dev(rows((S, gamma + 1, Hkv, 128), 201)), bf16_dev(rows((S, gamma + 1, Hkv, 128), 202))
    q = bf16_dev(rows((S, gamma + 1, Hq, 128), 203))
    acc = i32_dev([1, 3])

    class State:
        def __init__(self):
            self.dev, self.lens = to_dev(cache), i32_dev(L0)
            self.idx = torch.full((S, Hkv, 100), -1, dtype=torch.int32, device="cuda")
            self.idx[:, :, :60] = torch.arange(60, dtype=torch.int32, device="cuda")
            self.nsel = i32_dev([60, 60])
            self.base_l, self.base_n = self.lens.clone(), self.nsel.clone()
            self.draft, self.ver = torch.empty((S, Hq, 128), dtype=torch.bfloat16, device="cuda"), torch.empty_like(q)
            self.q0 = q[:, 0].contiguous()
            self.read = tuple(torch.empty((S, Hkv, 7, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.ws = bd.Workspace()

        def round(self):
            self.base_l.copy_(self.lens)
            self.base_n.copy_(self.nsel)
            bd.bd_cache_append_q(self.dev, self.lens, kn, vn, idx=self.idx, nsel=self.nsel)
            bd.bd_sparse_decode_attn_q(self.dev, self.q0, self.idx, self.nsel, self.lens, out=self.draft, workspace=self.ws)
            bd.bd_verify_attn_q(self.dev, q, self.lens, out=self.ver, workspace=self.ws)
            bd.bd_cache_read_q(self.dev, self.lens, 7, first=self.base_l, outputs=self.read)
            bd.bd_cache_rollback(self.lens, acc, gamma + 1, nsel=self.nsel, base_lens=self.base_l, base_nsel=self.base_n)

        def bytes(self):
            return [t.view(torch.uint8) for t in (*self.dev, self.lens, self.idx, self.nsel, self.draft, self.ver, *self.read)]

    case(f"captured round bits={bits}")
    eager, captured = State(), State()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured.round()                                     # sizes the workspace
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured.round()
    eager.round()
    for _ in range(4):
        g.replay()
        torch.cuda.synchronize()
        eager.round()
        torch.cuda.synchronize()
        for a, b in zip(captured.bytes(), eager.bytes()):
            assert torch.equal(a, b)


@BITS
@pytest.mark.parametrize("page", [0, 16])
def test_speculative_rounds_over_quantised_caches(bits, page):
    """Prefill, selection on the read-back keys, then rounds of drafts, verification, acceptance and rollback, all on
    quantised caches: caches and lengths follow the oracle byte by byte, attention within its bound."""
    S, Hq, Hkv, cap, gamma, W, B, V = 2, 8, 2, 400, 3, 16, 64, 997
    g = np.random.default_rng(170)
    prompt = [300, 211]
    n0 = max(prompt)
    kp, vp = rows((S, n0, Hkv, 128), 171), rows((S, n0, Hkv, 128), 172)
    zeros = tuple(np.zeros((S, Hkv, cap, w), np.uint8) for w in (16 * bits, 16 * bits, 4, 4))
    oc, ol = O.cache_append_q(zeros, [0, 0], kp, vp, bits, counts=prompt)
    table = None
    if page:
        width = cap // page
        table_h = g.permutation(S * width).astype(np.int32).reshape(S, width)
        dev = bd.quant_kv_empty(S * width, Hkv, page, bits)
        for b in dev:
            b.zero_()
        table = i32_dev(table_h)
    else:
        dev = to_dev(zeros)
    logical = (lambda: tuple(np.stack([np.concatenate([b[p] for p in table_h[s]], axis=1) for s in range(S)])
                             for b in to_host(dev))) if page else (lambda: to_host(dev))
    lens, kw = i32_dev([0, 0]), dict(page_table=table, max_seq_len=cap)
    case(f"rounds bits={bits} page={page}: prefill")
    bd.bd_cache_append_q(dev, lens, bf16_dev(kp), bf16_dev(vp), counts=i32_dev(prompt), **kw)
    k16, _ = bd.bd_cache_read_q(dev, lens, cap, with_v=False, **kw)
    qw = rows((S, W, Hq, 128), 173)
    idx0, nsel, _ = bd.bd_select_kv(k16, bf16_dev(qw), lens, B, return_scores=True)
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(logical(), oc))
    idx = torch.full((S, Hkv, B + 40), -1, dtype=torch.int32, device="cuda")
    idx[:, :, :B] = idx0
    oi, on = idx.cpu().numpy(), nsel.cpu().numpy()
    vals = lambda c: (values_as_bits(c[0], c[2], bits), values_as_bits(c[1], c[3], bits))
    for r in range(3):
        base_l, base_n, ob_l, ob_n = lens.clone(), nsel.clone(), ol.copy(), on.copy()
        for i in range(gamma + 1):
            kn, vn = rows((S, 1, Hkv, 128), 1000 * r + i), rows((S, 1, Hkv, 128), 1000 * r + 100 + i)
            case(f"rounds: {r} draft {i}")
            bd.bd_cache_append_q(dev, lens, bf16_dev(kn), bf16_dev(vn), idx=idx, nsel=nsel, **kw)
            oc, ol, oi, on = O.cache_append_q(oc, ol, kn, vn, bits, None, oi, on)
            q = rows((S, Hq, 128), 1000 * r + 200 + i)
            out, lse = bd.bd_sparse_decode_attn_q(dev, bf16_dev(q), idx, nsel, lens, return_lse=True, **kw)
            torch.cuda.synchronize()
            kb, vb = vals(oc)
            ref = lambda q, k, v: O.sparse_decode_attn(k, v, q, oi, on, ol)
            check_out(out, lse, *ref(q, kb, vb), kb, vb, q, ref, int(on.max()), f"draft {r} {i}")
        q = rows((S, gamma + 1, Hq, 128), 1000 * r + 300)
        out, lse = bd.bd_verify_attn_q(dev, bf16_dev(q), lens, return_lse=True, **kw)
        logits = g.standard_normal((S, gamma + 1, V)).astype(np.float32)
        draft = np.where(np.arange(gamma) < g.integers(0, gamma + 1, (S, 1)), logits.argmax(-1)[:, :gamma], 0).astype(np.int32)
        acc, _ = bd.bd_accept_len(torch.from_numpy(logits).cuda(), i32_dev(draft))
        bd.bd_cache_rollback(lens, acc, gamma + 1, nsel=nsel, base_lens=base_l, base_nsel=base_n)
        torch.cuda.synchronize()
        kb, vb = vals(oc)
        ref = lambda q, k, v: O.verify_attn(k, v, q, ol, gamma)
        check_out(out, lse, *ref(q, kb, vb), kb, vb, q, ref, int(max(ol)), f"verify {r}")
        oa = O.accept_len(logits, draft, gamma)[0]
        ol, on = O.cache_rollback(ol, oa, gamma + 1, nsel=on, base_lens=ob_l, base_nsel=ob_n)
        assert lens.cpu().tolist() == ol.tolist() and nsel.cpu().tolist() == on.tolist()
        assert all(np.array_equal(a, b) for a, b in zip(logical(), oc))
