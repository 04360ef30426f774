"""4-bit weights and cache without a GPU: the page format and the quantiser of the plain forms against each other, and
every refusal of the entry points that host-visible arguments allow."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2602_18447_amd import binding as cb
from tests import int4_ref as R
from tests.test_abi_cpu import _FakeDev, _cfg, _no_gpu_here


def test_pages_hold_every_element_once():
    kbit, vbit = R._places("cpu")
    both = torch.cat((kbit.reshape(-1), vbit.reshape(-1)))
    assert sorted(both.tolist()) == list(range(0, 8 * 2048, 4))
    assert cb.KV4_PAGE_BYTES == R.PAGE == 2048 + 2 * 16 * 4


@pytest.mark.parametrize("slot, is_v", [(0, False), (15, False), (3, True), (12, True)])
def test_a_row_written_is_the_row_read(slot, is_v):
    gen = torch.Generator().manual_seed(slot)
    pages = torch.full((2, 3, R.PAGE), 0x5A, dtype=torch.uint8)
    before = pages.clone()
    x = torch.randn(R.HD, generator=gen).bfloat16()
    c, s, z = R.quantise(x)
    R.write_row(pages, 1, 2, slot, c, s, z, is_v)
    got = R.read_pages(pages[1])[1 if is_v else 0]
    assert torch.equal(got[0][2, slot].long(), c) and got[1][2, slot] == s.double() and got[2][2, slot] == z.double()
    assert int((pages != before).sum()) <= 64 + 4 and torch.equal(pages[0], before[0])


def test_quantiser_of_the_plain_form():
    rows = torch.stack((torch.linspace(-3, 4, 128), torch.full((128,), 2.5), torch.zeros(128), torch.linspace(-1e6, 1e6, 128))).bfloat16()
    c, s, z = R.quantise(rows)
    back = z.double()[:, None] + s.double()[:, None] * c
    assert int(c[0].min()) == 0 and int(c[0].max()) == 15
    # half a step, and what s and z lose by being halves (2^-11 each; s over 15 steps)
    assert float((back[0] - rows[0].double()).abs().max()) <= 0.5 * float(s[0]) + 15 * 2.0 ** -11 * float(s[0]) + 2.0 ** -11 * 3
    assert torch.equal(back[1], rows[1].double()) and torch.equal(back[2], rows[2].double())
    assert float(back[3].abs().max()) <= 65504 * (1 + 2.0 ** -10)


class _Args:
    """Arguments of a valid call on made-up addresses; every test changes one of them."""

    def __init__(self, dtype="bf16", S=(3, 1), L=(40, 0), **cfg):
        self.ctx = cb.confspec_create(_cfg(dtype, **cfg))
        self.cu = np.concatenate([[0], np.cumsum(S)]).astype(np.int32)
        self.lens = np.asarray(L, dtype=np.int32)
        d = _FakeDev()
        self.batch, self.keep = cb.make_batch(d, d, d, self.cu, self.lens)
        self.kv = cb.make_kv4(d, d, 8, 16, 4)
        self.dev = d

    def append(self, qkv=None, n=None, hn=None, q=None, k=None, v=None, layer=0, stride=1024):
        d = self.dev
        return cb.confspec_op_kv4_append(self.ctx, self.kv, self.batch, layer, qkv or d, n, hn, q or d, k or d, v or d, qkv_stride=stride, stream=1)

    def read(self, k=None, layer=0):
        return cb.confspec_op_kv4_read(self.ctx, self.kv, self.batch, layer, k or self.dev, self.dev, stream=1)

    def attn(self, q=None, out=None, layer=0, scratch=None):
        d = self.dev
        return cb.confspec_op_kv4_attention(self.ctx, self.kv, self.batch, layer, q or d, d, d, out or d, scratch or d, stream=1)


def _refused(code, call, *a, **kw):
    with pytest.raises(cb.ConfSpecError) as e:
        call(*a, **kw)
    assert e.value.code == code, str(e.value)


class _Null:
    def data_ptr(self):
        return None

    def numel(self):
        return 0

    def element_size(self):
        return 1


def test_cache_operators_refuse_bad_arguments():
    _no_gpu_here()
    odd, null = _FakeDev(0x10008), _Null()
    a = _Args()
    for call in (a.append, a.read, a.attn):
        _refused(cb.E_INVALID_ARG, call, layer=2)
        _refused(cb.E_INVALID_ARG, call, layer=-1)
        for field, value, code in (("n_blocks", 0, cb.E_INVALID_ARG), ("block_size", 32, cb.E_UNSUPPORTED), ("block_size", 0, cb.E_UNSUPPORTED),
                                   ("max_blocks_per_seq", 0, cb.E_INVALID_ARG), ("pages", None, cb.E_INVALID_ARG), ("pages", 0x10008, cb.E_INVALID_ARG),
                                   ("block_table", None, cb.E_INVALID_ARG), ("max_blocks_per_seq", 2, cb.E_OUT_OF_RANGE)):
            keep = getattr(a.kv, field)
            setattr(a.kv, field, value)
            _refused(code, call)
            setattr(a.kv, field, keep)
    for kw in (dict(qkv=null), dict(q=null), dict(k=null), dict(v=null), dict(qkv=odd), dict(q=odd), dict(k=odd), dict(v=odd), dict(stride=1020),
               dict(stride=1022 + 4), dict(n=_FakeDev()), dict(hn=np.array([1, 1], dtype=np.int32))):
        _refused(cb.E_INVALID_ARG, a.append, **kw)
    for hn in ([4, 1], [-1, 0], [0, 2]):
        _refused(cb.E_OUT_OF_RANGE, a.append, n=_FakeDev(), hn=np.array(hn, dtype=np.int32))
    _refused(cb.E_INVALID_ARG, a.read, k=null)
    _refused(cb.E_INVALID_ARG, a.read, k=odd)
    _refused(cb.E_INVALID_ARG, a.attn, q=null)
    _refused(cb.E_INVALID_ARG, a.attn, out=odd)
    # rows behind the block table's end: written and read ones are refused, a suffix that is not stored is not
    full = _Args(S=(3, 1), L=(62, 0))
    _refused(cb.E_OUT_OF_RANGE, full.append)
    _refused(cb.E_OUT_OF_RANGE, full.read)
    _refused(cb.E_OUT_OF_RANGE, full.append, n=_FakeDev(), hn=np.array([3, 1], dtype=np.int32))
    # positions that would pass 31 bits
    far = _Args(S=(5, 1), L=(2 ** 31 - 1000, 0))
    far.kv.max_blocks_per_seq = 2 ** 27
    for call in (far.append, far.read, far.attn):
        _refused(cb.E_OUT_OF_RANGE, call)
    _refused(cb.E_OUT_OF_RANGE, cb.confspec_op_kv4_attention_scratch_bytes, far.ctx, far.batch)
    f32 = _Args("fp32")
    for call in (f32.append, f32.read, f32.attn):
        _refused(cb.E_UNSUPPORTED, call)
    _refused(cb.E_UNSUPPORTED, cb.confspec_op_kv4_attention_scratch_bytes, f32.ctx, f32.batch)
    for x in (a, full, far, f32):
        cb.confspec_destroy(x.ctx)


def test_host_counts_are_read_where_they_are_or_copied():
    a = np.arange(5, dtype=np.int32)
    address, keep = cb._host_i32(a, 5)
    assert address == a.ctypes.data and keep is a
    frozen = a.copy()
    frozen.setflags(write=False)
    for other in (frozen, np.arange(10, dtype=np.int32)[::2], a.astype(np.int64), a.astype(">i4"), [0, 1, 2, 3, 4], (7,)):
        address, keep = cb._host_i32(other, len(other))
        assert keep.dtype == np.int32 and keep.dtype.isnative and keep.flags.c_contiguous and address == keep.ctypes.data
        assert keep.tolist() == list(other)
    for short in (a[:4], a[:0], [1, 2, 3, 4], [1] * 6):
        with pytest.raises(ValueError):
            cb._host_i32(short, 5)


@pytest.mark.parametrize("S, L", [((1,), (100000,)), ((1, 1, 1), (0, 5, 70000)), ((300,), (40000,)), ((7,) * 40, (3000,) * 40)])
def test_attention_refuses_too_small_scratch(S, L):
    _no_gpu_here()
    a = _Args(S=S, L=L, n_q_heads=12)
    a.kv.max_blocks_per_seq = 1 << 14
    need = cb.confspec_op_kv4_attention_scratch_bytes(a.ctx, a.batch)
    if need:
        _refused(cb.E_WORKSPACE, a.attn, scratch=_FakeDev(0x10000, need - 1))
        _refused(cb.E_WORKSPACE, a.attn, scratch=_FakeDev(0x10010, need))
        _refused(cb.E_INVALID_ARG, a.attn, scratch=_Null())
    cb.confspec_destroy(a.ctx)


def test_weight_sizes_and_refusals():
    _no_gpu_here()
    assert cb.confspec_w4_bytes(32, 256, 128) == 2 * 2 * 1088
    assert cb.confspec_w4_bytes(16, 160, 32) == 2 * 1280            # the last record is filled up
    for N, K, g in ((8, 128, 128), (24, 128, 128), (0, 128, 128), (16, 64, 128), (16, 128, 16), (16, 128, 0), (16, 0, 32), (16, 96, 64), (-16, 128, 32)):
        assert cb.confspec_w4_bytes(N, K, g) == 0
    ctx, f32, d, odd = cb.confspec_create(_cfg()), cb.confspec_create(_cfg("fp32")), _FakeDev(), _FakeDev(0x10008)
    ok = dict(codes=d, scales=d, zeros=None, N=32, K=256, group=64, dst=d)
    pack = lambda ctx=ctx, **kw: cb.confspec_w4_pack(ctx, **{**ok, **kw}, stream=1)
    _refused(cb.E_UNSUPPORTED, pack, f32)
    _refused(cb.E_UNSUPPORTED, pack, N=24)
    _refused(cb.E_UNSUPPORTED, pack, group=48)
    _refused(cb.E_INVALID_ARG, pack, codes=_Null())
    _refused(cb.E_INVALID_ARG, pack, scales=_Null())
    _refused(cb.E_INVALID_ARG, pack, codes=_FakeDev(0x10002))
    _refused(cb.E_INVALID_ARG, pack, zeros=_FakeDev(0x10001))
    _refused(cb.E_WORKSPACE, pack, dst=_FakeDev(0x10080))
    _refused(cb.E_WORKSPACE, pack, dst=_FakeDev(0x10000, cb.confspec_w4_bytes(32, 256, 64) - 1))
    okg = dict(A=d, W4=d, residual=None, out=d, M=3, N=32, K=256, group=64, epilogue=cb.EPI_STORE_F32)
    gemm = lambda ctx=ctx, **kw: cb.confspec_op_w4_gemm(ctx, **{**okg, **kw}, stream=1)
    _refused(cb.E_UNSUPPORTED, gemm, f32)
    for kw in (dict(A=_Null()), dict(W4=_Null()), dict(out=_Null()), dict(A=odd), dict(out=odd), dict(W4=_FakeDev(0x10010)), dict(epilogue=3),
               dict(epilogue=-1), dict(residual=d), dict(epilogue=cb.EPI_RESID_F32), dict(M=0), dict(M=-3),
               dict(epilogue=cb.EPI_RESID_F32, residual=odd)):
        _refused(cb.E_INVALID_ARG, gemm, **kw)
    for kw in (dict(M=cb.W4_MAX_ROWS + 1), dict(N=40), dict(K=200), dict(group=16)):
        _refused(cb.E_UNSUPPORTED, gemm, **kw)
    cb.confspec_destroy(ctx)
    cb.confspec_destroy(f32)
    assert cb.lib.confspec_op_w4_gemm(None, None, None, None, None, 1, 16, 32, 32, 0, None) == cb.E_INVALID_ARG


@pytest.mark.parametrize("Hq, Hkv", [(12, 2), (40, 8), (64, 64), (128, 1)])
def test_attention_scratch_stays_small(Hq, Hkv):
    """Partial results are kept for at most about twice 2048 pieces of 32 rows, whatever the batch."""
    ctx = cb.confspec_create(_cfg(n_q_heads=Hq, n_kv_heads=Hkv))
    rng = np.random.default_rng(Hq)
    for _ in range(300):
        B = int(rng.choice([1, 2, 30, 256, 257, 900]))
        L = rng.integers(0, int(rng.choice([1, 100, 5000, 1 << 20, 1 << 30])) + 1, B).astype(np.int32)
        S = rng.integers(1, int(rng.choice([1, 8, 300, 4000])) + 1, B)
        cu = np.concatenate([[0], np.cumsum(S)]).astype(np.int32)
        d = _FakeDev()
        batch, keep = cb.make_batch(d, d, d, cu, L)
        assert cb.confspec_op_kv4_attention_scratch_bytes(ctx, batch) <= 2 * 2049 * 32 * 130 * 4, (B, L.max(), S.max())
    cb.confspec_destroy(ctx)


def test_weight_sizes_up_to_the_largest():
    """2^34 elements, K rounded up to whole records, and no more."""
    for N, K, group in ((1 << 17, 1 << 17, 128), (1 << 12, 1 << 22, 64), (1 << 27, 128, 32), (1 << 27, 32, 32), (1 << 17, (1 << 17) - 64, 64)):
        records = (N // 16) * ((K + 127) // 128)
        assert records == 1 << 23
        assert cb.confspec_w4_bytes(N, K, group) == records * (1024 + 64 * (128 // group))
        assert cb.confspec_w4_bytes(N + 16, K, group) == 0
    assert cb.confspec_w4_bytes(16, (1 << 22) + 128, 128) == 0
