"""Quantised caches on the CPU: the oracle's format against closed forms and torch's own conversions, the descriptor,
and every refusal of the C entry points and of the binding (nothing is launched: each call is refused on the host)."""
import ctypes
import os

import numpy as np
import pytest
import torch

import oracle as O
import paper_2606_00144_amd as bd
from quant_utils import bits_of, rows, special_rows

FAKE = 0x10000000
BITS = pytest.mark.parametrize("bits", [4, 8])


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(bd.library_path):
        from paper_2606_00144_amd import build
        build.build_library()
    return bd.lib()


# ------------------------------------------------------------------ the format

def test_grids():
    g8 = O.mx_grid(8)
    codes = torch.arange(127, dtype=torch.uint8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).float().numpy().astype(np.float64), g8)
    assert g8[-1] == 448 and g8[1] == 2.0 ** -9
    g4 = O.mx_grid(4)                                   # sign, two exponent bits of bias 1, one mantissa bit
    want = [m / 2 if k == 0 else (1 + m / 2) * 2.0 ** (k - 1) for k in range(4) for m in range(2)]
    assert g4.tolist() == want


def test_eight_bit_codes_are_those_of_torch():
    x = rows((300, 128), 1)
    c, s = O.mx_quantise(x, 8)
    y = O.bf16_to_f64(x) * np.repeat(2.0 ** (127 - s.astype(np.float64)), 32, axis=-1)
    t = torch.from_numpy(np.clip(y, -448, 448).astype(np.float32)).to(torch.float8_e4m3fn)
    assert np.array_equal(t.view(torch.uint8).numpy(), c)


@BITS
@pytest.mark.parametrize("a,step", [(1.0, 0), (1.75, 0), (1.7578125, 1), (1.8125, 1), (1.8203125, 2), (1.9921875, 2)])
def test_block_exponents(bits, a, step):
    # 1.75 (4 bits) and 1.8125 (8 bits) are the last maxima of their binade that keep its exponent
    x = np.zeros((1, 128), np.float32)
    x[0, ::32] = [a, -a, a * 2.0 ** 40, a * 2.0 ** -90]
    _, s = O.mx_quantise(bits_of(x), bits)
    up = int(step >= (1 if bits == 4 else 2))
    emax = 2 if bits == 4 else 8
    assert s[0].tolist() == [127 - emax + up, 127 - emax + up, 167 - emax + up, 37 - emax + up]


@BITS
def test_borders_of_the_format(bits):
    big = 3.3895314e38                                  # bf16's largest
    x = np.zeros((4, 128), np.float32)
    x[0, 0], x[0, 32], x[0, 64], x[0, 96] = big, -big, 2.0 ** -133, -2.0 ** -112
    x[1, 5], x[1, 40], x[1, 70] = np.nan, np.inf, -np.inf
    x[2, 3] = -0.0
    x[3, :32] = 1.0
    c, s = O.mx_quantise(bits_of(x), bits)
    v = O.mx_values(c, s, bits)
    top = 6.0 * 2.0 ** 125 if bits == 4 else 448.0 * 2.0 ** 119
    assert v[0, 0] == top and v[0, 32] == -top and v[0, 64] == 0.0
    assert v[0, 96] == -2.0 ** -112                     # 2^-111 times 0.5, the smallest 4-bit value
    assert s[1].tolist() == [255, 255, 255, 16] and np.isnan(v[1, :96]).all() and not v[1, 96:].any() and not c[1].any()
    assert np.signbit(v[2, 3]) and s[2].tolist() == [16] * 4
    assert (v[3, :32] == 1.0).all()


@BITS
def test_values_are_exact_in_bf16_and_quantise_to_themselves(bits):
    x = special_rows(500, 3)
    c, s = O.mx_quantise(x, bits)
    v = O.mx_values(c, s, bits)
    ok = ~np.isnan(v)
    b = bits_of(np.where(ok, v, 0.0))
    assert np.array_equal(O.bf16_to_f64(b), np.where(ok, v, 0.0))
    c2, s2 = O.mx_quantise(b, bits)
    assert np.array_equal(O.mx_values(c2, s2, bits), np.where(ok, v, 0.0))


@BITS
def test_rounding_is_to_the_nearest(bits):
    # brute force over the grid, every element of ordinary blocks; ties to the even code
    x = rows((60, 128), 4)
    c, s = O.mx_quantise(x, bits)
    v = O.mx_values(c, s, bits)
    grid = O.mx_grid(bits)
    two = np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, -1)
    y, q = np.abs(O.bf16_to_f64(x)) / two, np.abs(v) / two
    d = np.abs(y[..., None] - grid)
    assert np.array_equal(np.abs(y - q), d.min(-1))
    code = np.searchsorted(grid, q)
    tie = (d == d.min(-1, keepdims=True)).sum(-1) > 1
    assert tie.any() and (code[tie] % 2 == 0).all()


def test_append_oracle_against_a_plain_loop():
    S, Hkv, cap, n, bits = 2, 2, 9, 4, 4
    cache = tuple(np.full((S, Hkv, cap, w), 9, np.uint8) for w in (64, 64, 4, 4))
    kn, vn = rows((S, n, Hkv, 128), 5), rows((S, n, Hkv, 128), 6)
    idx = np.full((S, Hkv, 5), -1, np.int32)
    out, lens, oi, on = O.cache_append_q(cache, [7, 1], kn, vn, bits, [4, 3], idx, [1, 3])
    assert lens.tolist() == [9, 4] and on.tolist() == [3, 5]
    assert oi[0, 0].tolist() == [-1, 7, 8, -1, -1] and oi[1, 1].tolist() == [-1, -1, -1, 1, 2]
    for s, (a, b) in enumerate([(7, 9), (1, 4)]):
        for t in range(cap):
            for h in range(Hkv):
                if a <= t < b:
                    c, e = O.mx_quantise(vn[s, t - a, h], bits)
                    assert np.array_equal(out[1][s, h, t], c) and np.array_equal(out[3][s, h, t], e)
                else:
                    assert (out[1][s, h, t] == 9).all()


# ------------------------------------------------------------------ descriptor and refusals

def _cache(S=3, Hkv=2, rows_=24, bits=4):
    return bd.quant_kv_empty(S, Hkv, rows_, bits, device="cpu")


@BITS
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("layout", ["head", "token", "interleaved"])
def test_descriptor(bits, paged, layout):
    c = _cache(5, 2, 24, bits)
    if layout == "token":
        c = bd.QuantKV(*[b.transpose(1, 2).contiguous().transpose(1, 2) for b in c])
    elif layout == "interleaved":                       # K's and V's rows of a position side by side
        both, sc = torch.zeros(5, 2, 24, 2, 16 * bits, dtype=torch.uint8), torch.zeros(5, 2, 24, 2, 4, dtype=torch.uint8)
        c = bd.QuantKV(both[..., 0, :], both[..., 1, :], sc[..., 0, :], sc[..., 1, :])
    lens = torch.zeros(3 if paged else 5, dtype=torch.int32)
    table = torch.zeros(3, 4, dtype=torch.int32) if paged else None
    d = bd.qkv_desc(c, lens, table)
    for name in ("k", "v", "k_scale", "v_scale"):
        assert getattr(d, name) == getattr(c, name).data_ptr()
    w = 16 * bits
    st = [x // w for x in c.k.stride()]
    assert (d.bits, d.num_seqs, d.num_kv_heads, d.head_dim) == (bits, lens.shape[0], 2, 128)
    assert (d.stride_head, d.stride_tok) == (st[1], st[2]) and d.seq_lens == lens.data_ptr()
    if paged:
        assert (d.page_size, d.max_pages_per_seq, d.num_pages, d.stride_page, d.max_seq_len) == (24, 4, 5, st[0], 96)
        assert d.page_table == table.data_ptr()
    else:
        assert d.page_table is None and d.stride_seq == st[0] and d.max_seq_len == 24
    assert bd.qkv_desc(c, lens, table, 7).max_seq_len == 7


def test_descriptor_refusals():
    c, lens = _cache(), torch.zeros(3, dtype=torch.int32)
    wide = torch.zeros(3, 2, 24, 80, dtype=torch.uint8)[..., :64]                 # padded rows
    bad = [c._replace(k=c.k.int()), c._replace(k=c.k[..., :32]), c._replace(k=c.k[0]), c._replace(v=c.v[:, :, :8]),
           c._replace(k_scale=c.k_scale[..., :2]), c._replace(v_scale=c.v_scale.float()), c._replace(k=wide, v=wide),
           c._replace(k_scale=c.k_scale.transpose(1, 2).contiguous().transpose(1, 2),
                      v_scale=c.v_scale.transpose(1, 2).contiguous().transpose(1, 2)),
           bd.QuantKV(*[b.transpose(2, 3) for b in c])]
    for b in bad:
        with pytest.raises(bd.BdError):
            bd.qkv_desc(b, lens)
    for kw in (dict(seq_lens=lens.long()), dict(seq_lens=lens[:2]), dict(seq_lens=torch.zeros(6, dtype=torch.int32)[::2]),
               dict(page_table=lens), dict(page_table=torch.zeros(2, 2, dtype=torch.int32)),
               dict(page_table=torch.zeros(3, 8, dtype=torch.int32)[:, ::2]), dict(max_seq_len=25),
               dict(max_seq_len=2 ** 40, page_table=torch.zeros(3, 2, dtype=torch.int32))):
        with pytest.raises(bd.BdError):
            bd.qkv_desc(**dict(dict(cache=c, seq_lens=lens), **kw))
    with pytest.raises(bd.BdError):
        bd.quant_kv_empty(1, 1, 1, 16, device="cpu")


def test_tensors_off_the_gpu_are_refused():
    c, lens = _cache(), torch.zeros(3, dtype=torch.int32)
    rows_ = torch.zeros(3, 2, 2, 128, dtype=torch.bfloat16)
    idx, q = torch.zeros(3, 2, 4, dtype=torch.int32), torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    for call in (lambda: bd.bd_cache_append_q(c, lens, rows_, rows_), lambda: bd.bd_cache_read_q(c, lens, 4),
                 lambda: bd.bd_sparse_decode_attn_q(c, q, idx, lens, lens),
                 lambda: bd.bd_verify_attn_q(c, q[:, None].contiguous(), lens)):
        with pytest.raises(bd.BdError, match="current GPU"):
            call()


def test_binding_refusals():
    c, lens = _cache(), torch.zeros(3, dtype=torch.int32)
    rows_ = torch.zeros(3, 2, 2, 128, dtype=torch.bfloat16)
    idx, q = torch.zeros(3, 2, 4, dtype=torch.int32), torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    out = torch.zeros(3, 2, 4, 128, dtype=torch.bfloat16)
    bad = [lambda: bd.bd_cache_append_q(c, lens, rows_.float(), rows_), lambda: bd.bd_cache_append_q(c, lens, rows_, rows_[:, :1]),
           lambda: bd.bd_cache_append_q(c, lens, rows_[:2], rows_[:2]), lambda: bd.bd_cache_append_q(c, lens, rows_.transpose(1, 2), rows_),
           lambda: bd.bd_cache_append_q(c, lens, rows_, rows_, counts=lens[:2]), lambda: bd.bd_cache_append_q(c, lens, rows_, rows_, idx=idx),
           lambda: bd.bd_cache_append_q(c, lens, rows_, rows_, idx=idx[:, :1].contiguous(), nsel=lens),
           lambda: bd.bd_cache_read_q(c, lens, -1), lambda: bd.bd_cache_read_q(c, lens, 4, first=lens.long()),
           lambda: bd.bd_cache_read_q(c, lens, 4, outputs=(out[:, :, :3], None)), lambda: bd.bd_cache_read_q(c, lens, 4, outputs=(out.float(), None)),
           lambda: bd.bd_cache_read_q(c, lens, 4, outputs=(out, out.transpose(1, 2).contiguous().transpose(1, 2))),
           lambda: bd.bd_sparse_decode_attn_q(c, q.float(), idx, lens, lens), lambda: bd.bd_sparse_decode_attn_q(c, q[:2], idx, lens, lens),
           lambda: bd.bd_sparse_decode_attn_q(c, q, idx[:, :1].contiguous(), lens, lens), lambda: bd.bd_sparse_decode_attn_q(c, q, idx.long(), lens, lens),
           lambda: bd.bd_sparse_decode_attn_q(c, q, idx, lens[:2], lens), lambda: bd.bd_sparse_decode_attn_q(c, q, idx, lens, lens, out=out),
           lambda: bd.bd_cache_read_q(c, lens, 4, outputs=(out[:, :, :1].expand(3, 2, 4, 128), None)),
           lambda: bd.bd_cache_append_q(tuple(c), lens, rows_, rows_),
           lambda: bd.bd_cache_append_q(bd.QuantKV(*[b[:1].expand(3, -1, -1, -1) for b in c]), lens, rows_, rows_),
           lambda: bd.bd_verify_attn_q(c, q, lens), lambda: bd.bd_verify_attn_q(c, q[:2, None].contiguous(), lens),
           lambda: bd.bd_verify_attn_q(c, q[:, None, :, :64].contiguous(), lens)]
    for i, call in enumerate(bad):
        with pytest.raises(bd.BdError) as e:
            call()
        assert e.value.status == bd.BD_ERR_INVALID_ARG and "current GPU" not in str(e.value), i


def _kv(**over):
    d = bd.QkvDesc()
    d.k = d.v = d.k_scale = d.v_scale = d.seq_lens = FAKE
    d.bits, d.num_seqs, d.num_kv_heads, d.head_dim, d.max_seq_len = 4, 2, 8, 128, 4096
    d.stride_seq, d.stride_head, d.stride_tok = 8 * 4096, 4096, 1
    for k, v in over.items():
        setattr(d, k, v)
    return d


PAGED = dict(page_table=FAKE, page_size=16, max_pages_per_seq=256, num_pages=600, stride_page=128, stride_head=16)


def test_shared_rejections(L):
    ref = ctypes.byref
    calls = [lambda kv: L.bd_verify_attn_q(kv, FAKE, 32, 5, 0.1, FAKE, None, FAKE, 1 << 40, None),
             lambda kv: L.bd_sparse_decode_attn_q(kv, FAKE, 32, FAKE, 64, FAKE, 0.1, FAKE, None, FAKE, 1 << 40, None),
             lambda kv: L.bd_cache_append_q(kv, FAKE, FAKE, 1, None, None, 0, None, None),
             lambda kv: L.bd_cache_read_q(kv, None, 1, FAKE, FAKE, 0, 0, 0, None)]
    inv, uns = bd.BD_ERR_INVALID_ARG, bd.BD_ERR_UNSUPPORTED
    cases = [(dict(head_dim=64), uns), (dict(bits=6), uns), (dict(k=0), inv), (dict(v_scale=0), inv), (dict(k=FAKE + 8), inv),
             (dict(k_scale=FAKE + 2), inv), (dict(seq_lens=0), inv), (dict(num_seqs=0), inv), (dict(num_kv_heads=0), inv),
             (dict(max_seq_len=-1), inv), (dict(max_seq_len=(1 << 30) + 1, stride_tok=0), uns), (dict(stride_tok=-1), inv), (dict(stride_seq=-8), inv),
             (dict(stride_tok=(1 << 19) + 1), uns), (dict(stride_head=1 << 31), uns), (dict(stride_seq=1 << 40), uns),
             (dict(num_seqs=2 ** 21, num_kv_heads=16), uns), (dict(stride_seq=(1 << 31) - 1, stride_head=1), uns),
             (dict(PAGED, page_size=0), inv), (dict(PAGED, num_pages=0), inv), (dict(PAGED, max_pages_per_seq=255), inv),
             (dict(PAGED, stride_page=-1), inv), (dict(PAGED, stride_page=1 << 23), uns)]
    for call in calls:
        assert call(None) == inv
        for over, want in cases:
            assert call(ref(_kv(**over))) == want, over


def test_operation_rejections(L):
    ref, inv, uns = ctypes.byref, bd.BD_ERR_INVALID_ARG, bd.BD_ERR_UNSUPPORTED

    def ver(**a):
        g = lambda n, d: a.get(n, d)
        return L.bd_verify_attn_q(ref(g("kv", _kv())), g("q", FAKE), g("hq", 32), g("gamma", 5), g("scale", 0.1), g("out", FAKE),
                                  None, g("ws", FAKE), g("wsb", 1 << 40), None)
    for a in (dict(q=None), dict(q=FAKE + 8), dict(out=None), dict(out=FAKE + 2), dict(hq=30), dict(gamma=-1), dict(gamma=4096),
              dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert ver(**a) == inv, a
    assert ver(ws=None) == bd.BD_ERR_WORKSPACE and ver(ws=FAKE + 64) == bd.BD_ERR_WORKSPACE and ver(wsb=100) == bd.BD_ERR_WORKSPACE
    assert ver(kv=_kv(num_kv_heads=1), hq=2 ** 17) == uns
    need = L.bd_verify_attn_q_workspace_bytes(2, 8, 32, 5, 4096)
    assert ver(wsb=need - 1) == bd.BD_ERR_WORKSPACE

    def dec(**a):
        g = lambda n, d: a.get(n, d)
        return L.bd_sparse_decode_attn_q(ref(g("kv", _kv())), g("q", FAKE), g("hq", 32), g("idx", FAKE), g("ld", 64), g("nsel", FAKE),
                                         g("scale", 0.1), g("out", FAKE), None, g("ws", FAKE), g("wsb", 1 << 40), None)
    for a in (dict(q=None), dict(out=FAKE + 2), dict(idx=None), dict(ld=-1), dict(nsel=None), dict(scale=0.0), dict(hq=12)):
        assert dec(**a) == inv, a
    assert dec(ws=None) == bd.BD_ERR_WORKSPACE
    assert dec(ld=2 ** 31 - 1) == uns

    app = lambda **a: L.bd_cache_append_q(ref(a.get("kv", _kv())), a.get("k", FAKE), a.get("v", FAKE), a.get("n", 1), None,
                                          a.get("idx"), a.get("ld", 0), a.get("nsel"), None)
    assert app(n=0) == bd.BD_OK                                 # nothing to do, nothing launched
    for a in (dict(n=-1), dict(k=None), dict(v=FAKE + 8), dict(idx=FAKE), dict(nsel=FAKE), dict(idx=FAKE, nsel=FAKE, ld=-1)):
        assert app(**a) == inv, a
    assert app(n=2 ** 30 + 1) == uns

    rd = lambda **a: L.bd_cache_read_q(ref(a.get("kv", _kv())), None, a.get("n", 1), a.get("k", FAKE), a.get("v", FAKE),
                                       a.get("ss", 0), a.get("sh", 0), a.get("st", 0), None)
    assert rd(n=0) == bd.BD_OK
    for a in (dict(n=-1), dict(k=None, v=None), dict(k=FAKE + 8), dict(ss=-8), dict(sh=4), dict(st=129)):
        assert rd(**a) == inv, a
    assert rd(n=2 ** 30 + 1) == uns
    assert rd(kv=_kv(v=0, v_scale=0)) == inv                    # V is asked for


def test_workspace_sizes(L):
    v, d = L.bd_verify_attn_q_workspace_bytes, L.bd_sparse_decode_attn_q_workspace_bytes
    assert v(8, 8, 32, 5, 16384) % 256 == 0 and v(8, 8, 32, 5, 16384) > 1 << 20
    # scratch follows the launch, not the batch or the context
    assert v(64, 32, 32, 5, 16384) == v(64, 32, 32, 5, 131072) == v(1, 32, 32, 5, 131072)
    assert d(64, 32, 32, 2048) <= 1 << 25
    assert v(0, 8, 32, 5, 4096) == 0 and v(8, 8, 32, 4096, 4096) == 0 and v(8, 8, 30, 5, 4096) == 0 and v(8, 8, 32, 5, -1) == 0
    assert d(8, 8, 32, -1) == 0 and d(8, 1, 2 ** 17, 64) == 0
    assert v(1, 1, 1, 0, 0) > 0 and d(1, 1, 1, 0) > 0
