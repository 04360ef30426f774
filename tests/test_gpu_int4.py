"""Products with 4-bit weights, the append to a 4-bit paged cache, its rows read back and the attention over it, against
plain forms in 64 bits (tests/int4_ref.py, which derives the bounds)."""
import math

import numpy as np
import pytest
import torch

from paper_2602_18447_amd import binding as cb
from tests import int4_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA = 1.0e6


class Ctx:
    def __init__(self, Hq=4, Hkv=2, n_layers=1, theta=THETA):
        self.ptr = cb.confspec_create(cb.make_model_cfg(n_layers, 128 * Hq, Hq, Hkv, 128, 256, 1024, theta, 1e-6, "bf16"), 0)

    def __enter__(self):
        return self.ptr

    def __exit__(self, *exc):
        torch.cuda.synchronize()
        cb.confspec_destroy(self.ptr)


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


class Cache:
    """Batch, block table (pages dealt out by a permutation) and, unless given, a filled cache."""

    def __init__(self, gen, Hkv, L, S, n_layers=1, pages=None, spare=2, cover_suffix=True):
        self.L, self.S = list(L), list(S)
        need = [max(1, (l + (s if cover_suffix else 0) + 15) // 16) for l, s in zip(L, S)]
        self.n_blocks = sum(need) + spare
        order = torch.randperm(self.n_blocks, generator=gen, device=DEV).cpu().numpy().astype(np.int32)
        self.table = np.full((len(need), max(need)), 2 ** 30, dtype=np.int32)        # (entries that are never looked at)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        self.pages = R.random_pages(gen, n_layers, self.n_blocks, Hkv, DEV) if pages is None else pages
        self.cu = np.concatenate([[0], np.cumsum(S)]).astype(np.int32)
        self.lens = np.asarray(L, dtype=np.int32)
        self.T = int(self.cu[-1])
        dev = [torch.from_numpy(x).to(DEV) for x in (self.table, self.cu, self.lens)]
        self.ids = torch.zeros(self.T, dtype=torch.int32, device=DEV)
        self.kv = cb.make_kv4(self.pages, dev[0], self.n_blocks, 16, self.table.shape[1])
        self.batch, keep = cb.make_batch(self.ids, dev[1], dev[2], self.cu, self.lens)
        self.keep = (dev, keep)

    def poison(self, layer=None):
        """Every row that no trace sees becomes bytes 0xFF: codes 15, s and z not a number."""
        seen = torch.zeros(self.pages.shape[1], 16, dtype=torch.bool, device=DEV)
        for b, l in enumerate(self.L):
            j = torch.arange(l, device=DEV)
            seen[torch.from_numpy(self.table[b].astype(np.int64)).to(DEV)[j // 16], j % 16] = True
        kbit, vbit = R._places(DEV)
        flat = self.pages.view(-1, self.pages.shape[1], self.pages.shape[2], R.PAGE)
        for slot in range(16):
            blocks = torch.nonzero(~seen[:, slot]).view(-1)
            for bits in (kbit, vbit):
                for half in (0, 4):
                    at = bits[slot][bits[slot] % 8 == half] // 8
                    page = flat[:, blocks]
                    page[..., at] |= 0xF << half
                    flat[:, blocks] = page
            page = flat[:, blocks]
            page[..., 2048 + 4 * slot:2052 + 4 * slot] = 0xFF
            page[..., 2112 + 4 * slot:2116 + 4 * slot] = 0xFF
            flat[:, blocks] = page

    def scratch(self, ctx):
        n = cb.confspec_op_kv4_attention_scratch_bytes(ctx, self.batch)
        return torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device=DEV)


# ---------------------------------------------------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------------------------------------------------
def _w4_case(M, N, K, group, epi, seed, zeros=True, scale_a=1.0):
    gen = _gen(seed)
    codes, s, z, w = R.w4_quantise_case(gen, N, K, group, DEV, zeros)
    a = (torch.randn(M, K, generator=gen, device=DEV) * scale_a).bfloat16()
    resid = torch.randn(M, N, generator=gen, device=DEV) if epi == cb.EPI_RESID_F32 else None
    packed = torch.full((cb.confspec_w4_bytes(N, K, group),), 0xFF, dtype=torch.uint8, device=DEV)
    n_out = N // 2 if epi == cb.EPI_SWIGLU else N
    # guard elements behind the result: they stay as they were
    out = torch.full((M * n_out + 64,), 7.0, dtype=torch.bfloat16 if epi == cb.EPI_SWIGLU else torch.float32, device=DEV)
    with Ctx() as ctx:
        cb.confspec_w4_pack(ctx, codes, s, z, N, K, group, packed, gate_up=epi == cb.EPI_SWIGLU)
        cb.confspec_op_w4_gemm(ctx, a, packed, resid, out, M, N, K, group, epi)
        first = out.clone()
        cb.confspec_op_w4_gemm(ctx, a, packed, resid, out, M, N, K, group, epi)
    assert torch.equal(first, out), "a product of the same operands comes out the same"
    assert bool((out[M * n_out:] == 7.0).all())
    y, tol = R.w4_gemm(a, w, s, z, group)
    if epi == cb.EPI_SWIGLU:
        y, tol = R.swiglu(y, tol)
    elif epi == cb.EPI_RESID_F32:
        y = y + resid.double()
        tol = tol + 2.0 ** -24 * y.abs()
    err = (out[:M * n_out].double().view(M, n_out) - y).abs()
    print(f"w4 M {M} N {N} K {K} group {group} epi {epi}: {float((err / tol).max()):.3f} of the bound", flush=True)
    assert bool((err <= tol).all())


@pytest.mark.parametrize("M", [1, 2, 3, 8, 15, 16, 17, 31, 32, 33, 48, 64, 65, 100, 127, 128])
@pytest.mark.parametrize("N, K, group, epi", [(256, 512, 128, 0), (144, 1600, 64, 1), (48, 416, 32, 2)])
def test_w4_rows(M, N, K, group, epi):
    _w4_case(M, N, K, group, epi, 100 * M + N)


@pytest.mark.parametrize("N, K, group", [(16, 32, 32), (16, 64, 64), (16, 128, 128), (32, 96, 32), (16, 8960, 64), (1536, 1536, 128), (2048, 160, 32),
                                         (5120, 27648, 64), (17920, 1536, 128), (80, 11008, 32), (4112, 2176, 64), (16, 32768, 128)])
@pytest.mark.parametrize("M, epi", [(1, 0), (5, 2), (20, 1), (70, 2)])
def test_w4_shapes(N, K, group, M, epi):
    _w4_case(M, N, K, group, epi, N + K + M)


@pytest.mark.parametrize("M, N", [(20, 5136), (32, 4112), (17, 8208), (64, 10256), (40, 4144), (33, 8208), (90, 7200), (100, 6160), (128, 12304), (70, 2576), (33, 2320)])
@pytest.mark.parametrize("K, group, epi", [(416, 32, 0), (1088, 64, 1), (640, 128, 2)])
def test_w4_many_rows_on_wide_matrices(M, N, K, group, epi):
    """Every tile that more than 16 rows can take."""
    _w4_case(M, N, K, group, epi, 9)


@pytest.mark.parametrize("M", [1, 40])
def test_w4_zero_points_of_eight_when_none_are_given(M):
    _w4_case(M, 272, 640, 128, cb.EPI_STORE_F32, 5, zeros=False)


@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_w4_activations_of_any_size(scale):
    _w4_case(7, 64, 512, 64, cb.EPI_STORE_F32, 6, scale_a=scale)


@pytest.mark.parametrize("M", [4, 90])
def test_w4_residual_in_place_and_a_row_that_is_not_finite(M):
    """An infinity or NaN in one row of activations stays in that row."""
    N, K, g = 192, 768, 128
    gen = _gen(8)
    codes, s, z, w = R.w4_quantise_case(gen, N, K, g, DEV)
    a = torch.randn(M, K, generator=gen, device=DEV).bfloat16()
    bad = a.clone()
    bad[1, 5], bad[3, 700] = float("inf"), float("nan")
    packed = torch.empty(cb.confspec_w4_bytes(N, K, g), dtype=torch.uint8, device=DEV)
    x0 = torch.randn(M, N, generator=gen, device=DEV)
    with Ctx() as ctx:
        cb.confspec_w4_pack(ctx, codes, s, z, N, K, g, packed)
        outs = []
        for act in (a, bad):
            x = x0.clone()
            cb.confspec_op_w4_gemm(ctx, act, packed, x, x, M, N, K, g, cb.EPI_RESID_F32)
            outs.append(x)
    y, tol = R.w4_gemm(a, w, s, z, g)
    y = y + x0.double()
    assert bool(((outs[0].double() - y).abs() <= tol + 2.0 ** -24 * y.abs()).all())
    rest = [i for i in range(M) if i not in (1, 3)]
    assert torch.equal(outs[1][rest], outs[0][rest])
    assert not bool(torch.isfinite(outs[1][1]).any()) and bool(torch.isnan(outs[1][3]).all())


# ---------------------------------------------------------------------------------------------------------------------
# append and read
# ---------------------------------------------------------------------------------------------------------------------
def _append_case(Hq, Hkv, L, S, n_append, seed, layer=0, n_layers=1, pad=0, theta=THETA, edit=None):
    gen = _gen(seed)
    c = Cache(gen, Hkv, L, S, n_layers=n_layers)
    width = (Hq + 2 * Hkv) * 128
    buf = torch.randn(c.T, width + pad, generator=gen, device=DEV)
    if edit:
        edit(buf[:, :width].view(c.T, Hq + 2 * Hkv, 128), Hq, Hkv)
    q = torch.empty(c.T, Hq, 128, dtype=torch.bfloat16, device=DEV)
    k = torch.empty(c.T, Hkv, 128, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    want = c.pages.clone()
    hn = None if n_append is None else np.asarray(n_append, dtype=np.int32)
    dn = None if hn is None else torch.from_numpy(hn).to(DEV)
    kr, vr = (torch.empty(c.T, Hkv, 128, device=DEV) for _ in range(2))
    with Ctx(Hq, Hkv, n_layers, theta) as ctx:
        cb.confspec_op_kv4_append(ctx, c.kv, c.batch, layer, buf, dn, hn, q, k, v, qkv_stride=width + pad)
        cb.confspec_op_kv4_read(ctx, c.kv, c.batch, layer, kr, vr)
    x = buf[:, :width].view(c.T, Hq + 2 * Hkv, 128)
    pos = torch.from_numpy(np.concatenate([l + np.arange(s) for l, s in zip(L, S)])).to(DEV)
    rot = R.rotate(x[:, :Hq + Hkv], pos, theta)
    # rounded to fp32, then to bf16: half a step each
    for got, ref in ((q, rot[:, :Hq]), (k, rot[:, Hq:]), (v, x[:, Hq + Hkv:].double())):
        fin = torch.isfinite(ref)
        assert bool(((got.double() - ref).abs()[fin] <= (2.0 ** -8 + 2.0 ** -24) * ref.abs()[fin] + 2.0 ** -133).all())
    n = list(S) if n_append is None else list(n_append)
    kc, ks, kz = (y.cpu() for y in R.quantise(k))
    vc, vs, vz = (y.cpu() for y in R.quantise(v))
    want, have = want.cpu(), c.pages.cpu()
    for b in range(len(L)):
        for i in range(n[b]):
            t, row = int(c.cu[b]) + i, L[b] + i
            for h in range(Hkv):
                blk = int(c.table[b, row // 16])
                R.write_row(want[layer], blk, h, row % 16, kc[t, h], ks[t, h], kz[t, h], False)
                R.write_row(want[layer], blk, h, row % 16, vc[t, h], vs[t, h], vz[t, h], True)
    assert torch.equal(want, have), "the rows named, and no other byte"
    pages = have[layer].view(-1, R.PAGE)
    (kc, ks, kz), (vc, vs, vz) = R.read_pages(pages)
    for got, (cc, ss, zz) in ((kr.cpu(), (kc, ks, kz)), (vr.cpu(), (vc, vs, vz))):
        vals = (zz[..., None] + ss[..., None] * cc).float().view(c.n_blocks, Hkv, 16, 128)      # one rounding
        for b in range(len(L)):
            row = L[b] + torch.arange(S[b])
            blk = torch.from_numpy(c.table[b].astype(np.int64))[row // 16]
            assert torch.equal(got[int(c.cu[b]):int(c.cu[b + 1])], vals[blk, :, row % 16])


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (12, 2), (40, 8), (6, 3), (7, 7), (34, 2)])
@pytest.mark.parametrize("L, S, n", [((0,), (1,), None), ((17, 0, 31), (1, 1, 1), None), ((5, 160, 63), (20, 33, 1), (20, 0, 1)), ((100, 3), (1, 70), (0, 69))])
def test_append_and_read(Hq, Hkv, L, S, n):
    _append_case(Hq, Hkv, L, S, n, 31 * Hq + sum(L))


def test_append_many_traces_of_one_token():
    rng = np.random.default_rng(3)
    _append_case(4, 2, [int(x) for x in rng.integers(0, 400, 150)], [1] * 150, None, 77)


def test_append_in_another_layer_with_rows_that_lie_apart():
    _append_case(4, 2, (30, 2), (5, 9), (5, 4), 78, layer=2, n_layers=3, pad=132)


@pytest.mark.parametrize("theta", [1.0e4, 5.0e5])
def test_append_at_far_positions(theta):
    """Angles of positions beyond 2^17 need more than fp32 has."""
    _append_case(2, 1, (200000, 131071), (3, 18), None, 79, theta=theta)


def test_append_elements_next_to_a_tie():
    """Rows from 2^-k to a half's largest values, whose elements lie near (c + 1/2) s: codes as the exact quotient has them."""
    def edit(x, Hq, Hkv):
        gen = _gen(45)
        n = x.shape[0] * Hkv
        lo = -(2.0 ** torch.randint(-14, 4, (n, 1), generator=gen, device=DEV)) * (1 + torch.randint(0, 128, (n, 1), generator=gen, device=DEV) / 128.0)
        hi = 2.0 ** torch.randint(-8, 12, (n, 1), generator=gen, device=DEV) * (1 + torch.randint(0, 128, (n, 1), generator=gen, device=DEV) / 128.0)
        v = lo + (hi - lo) * (torch.randint(0, 15, (n, 128), generator=gen, device=DEV) + 0.5) / 15.0
        v[:, :1], v[:, 1:2] = lo, hi
        x[:, Hq + Hkv:] = v.view(-1, Hkv, 128)
    _append_case(4, 4, (9, 0), (150, 90), None, 46, edit=edit)


def test_append_rows_of_every_kind():
    _append_case(3, 3, (13,), (12,), None, 80, edit=_edit_values)


def _edit_values(x, Hq, Hkv):
    """Values of every kind; of keys only what the rotation leaves finite."""
    kv = x[:, Hq:]
    v = x[:, Hq + Hkv:]
    kv[0] = 0.0                                                # s is 0
    kv[1] = -2.5
    kv[2] *= 1e-6                                              # s below the normal halves
    kv[3] *= 3e4                                               # beyond the halves: clamped
    v[4, :, 7] = float("inf")
    v[5, :, 9] = -float("inf")
    kv[6] = 100.0 + kv[6] * 1e-3                               # all values near a far one
    kv[7] = kv[7].sign()
    v[8] = torch.arange(128, device=x.device) % 16 * 0.5       # values on codes, and in the middle between two
    v[9] = torch.arange(128, device=x.device) % 31 * 0.25 - 2


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
def _attn_check(ctx, c, Hq, Hkv, q, k, v, layer=0, stream=None):
    out = torch.full((c.T * Hq * 128 + 64,), 7.0, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, layer, q, k, v, out, c.scratch(ctx))
    torch.cuda.synchronize()
    assert bool((out[c.T * Hq * 128:] == 7.0).all())
    got = out[:c.T * Hq * 128].view(c.T, Hq * 128)
    ref, tol = R.attention(c.pages[layer], c.table, q, k, v, c.cu, c.lens, Hq, Hkv)
    err = (got.double() - ref).abs()
    print(f"attention {Hq}/{Hkv} L {c.L[:6]} S {c.S[:6]}: {float((err / tol).max()):.3f} of the bound", flush=True)
    assert bool((err <= tol).all())
    return got


def _attn_case(Hq, Hkv, L, S, seed, q_scale=1.0, layer=0, n_layers=1, poison=True, **cache):
    gen = _gen(seed)
    c = Cache(gen, Hkv, L, S, n_layers=n_layers, **cache)
    if poison:
        c.poison()
    q = (torch.randn(c.T, Hq, 128, generator=gen, device=DEV) * q_scale).bfloat16()
    k = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    v = (torch.randn(c.T, Hkv, 128, generator=gen, device=DEV) * 0.5).bfloat16()
    with Ctx(Hq, Hkv, n_layers) as ctx:
        return _attn_check(ctx, c, Hq, Hkv, q, k, v, layer)


@pytest.mark.parametrize("L", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 511, 1000, 2048, 5003])
@pytest.mark.parametrize("S", [1, 2, 5, 33])
def test_attention_lengths(L, S):
    _attn_case(12, 2, (L,), (S,), L + S)


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (2, 1), (5, 1), (8, 1), (3, 3), (16, 1), (17, 1), (34, 2), (40, 8), (64, 1), (100, 1)])
@pytest.mark.parametrize("L, S", [((300,), (1,)), ((77, 0, 530), (3, 16, 1)), ((40,), (65,))])
def test_attention_heads(Hq, Hkv, L, S):
    _attn_case(Hq, Hkv, L, S, Hq * 7 + len(L))


@pytest.mark.parametrize("seed", range(6))
def test_attention_ragged_batches(seed):
    rng = np.random.default_rng(seed)
    B = int(rng.integers(2, 40))
    L = [int(x) for x in rng.integers(0, int(rng.choice([20, 300, 3000])), B)]
    S = [int(x) for x in rng.integers(1, int(rng.choice([2, 9, 70])) + 1, B)]
    Hq, Hkv = [(12, 2), (40, 8), (4, 4)][seed % 3]
    _attn_case(Hq, Hkv, L, S, seed)


@pytest.mark.parametrize("Hq, Hkv, L, S", [(40, 8, (0, 1, 16, 31, 33, 100, 290, 5), (60, 64, 33, 97, 128, 65, 64, 160)), (34, 2, (70,) * 12, tuple(range(30, 54, 2))),
                                           (4, 4, (0, 64, 200), (256, 300, 312)), (8, 8, (200,) * 40, (20, 65) * 20)])
def test_attention_many_rows_on_few_keys(Hq, Hkv, L, S):
    _attn_case(Hq, Hkv, L, S, 18)


@pytest.mark.parametrize("L, S", [((40000,), (1,)), ((150000, 70000), (1, 5)), ((20000, 5), (2, 3)), ((9000,), (150,)), ((0, 10), (400, 300))])
def test_attention_long(L, S):
    _attn_case(6, 1, L, S, 11)


@pytest.mark.parametrize("Hq, Hkv, L, S", [(35, 1, (9600,), (128,)), (8, 8, (12000,) * 17, (1,) * 17), (64, 1, (27000,), (150,))])
def test_attention_wavefronts_with_more_than_32_chunks(Hq, Hkv, L, S):
    """Batches whose pieces are long: a wavefront's block numbers come in several rounds."""
    _attn_case(Hq, Hkv, L, S, 19, poison=False)


@pytest.mark.parametrize("q_scale", [0.0, 1e-3, 8.0, 60.0])
def test_attention_from_even_to_single_weights(q_scale):
    _attn_case(4, 2, (700, 33), (3, 1), 12, q_scale=q_scale)


def test_attention_queries_of_any_size():
    """Rows of q from 1e-30 to 1e30, elements of one row 2^20 apart, and a row of zeros: each as if alone."""
    gen = _gen(42)
    Hq, Hkv = 8, 2
    c = Cache(gen, Hkv, (150, 20), (4, 9))
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV)
    q = q * torch.tensor([1e-30, 1e-3, 1.0, 3.0, 0.0, 30.0, 1e10, 1e30], device=DEV)[:, None]
    q[:, 2, ::7] *= 2.0 ** -20
    k = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    v = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    with Ctx(Hq, Hkv) as ctx:
        out = _attn_check(ctx, c, Hq, Hkv, q.bfloat16(), k, v)
    assert bool(torch.isfinite(out).all())


def test_attention_in_another_layer():
    _attn_case(4, 2, (50, 120), (2, 1), 13, layer=2, n_layers=3)


def test_attention_where_the_block_table_ends_with_the_context():
    """The suffix needs no blocks of its own; the last page is full or not."""
    _attn_case(4, 2, (48, 33, 1), (20, 2, 5), 14, cover_suffix=False)


def test_attention_of_many_traces():
    rng = np.random.default_rng(9)
    _attn_case(2, 1, [int(x) for x in rng.integers(0, 60, 700)], [1 + int(x) for x in rng.integers(0, 2, 700)], 15)


@pytest.mark.parametrize("kind", ["constant", "zero", "tiny", "huge", "one_large"])
def test_attention_over_values_of_every_size(kind):
    gen = _gen(16)
    Hq, Hkv, L, S = 6, 2, (90, 400), (1, 4)
    c = Cache(gen, Hkv, L, S)
    n = c.pages[0].shape[0] * Hkv
    x = torch.randn(n, 16, 128, generator=gen, device=DEV)
    x = {"constant": x * 0 + 1.75, "zero": x * 0, "tiny": x * 1e-5, "huge": x * 1e4, "one_large": x}[kind]
    if kind == "one_large":
        x[:, 3] *= 2000.0
    vc, vs, vz = R.quantise(x.bfloat16())
    page = c.pages.view(n, R.PAGE)
    bit = R._places(DEV)[1]
    for half in (0, 4):
        at = bit[bit % 8 == half] // 8
        page[:, at] = (page[:, at] & (0xF0 if half == 0 else 0x0F)) | (vc[:, bit % 8 == half] << half).to(torch.uint8)
    page[:, 2112:2176] = torch.stack((vs, vz), -1).view(n, 32).contiguous().view(torch.uint8)
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV).bfloat16()
    k = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    v = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16() * 0.1
    with Ctx(Hq, Hkv) as ctx:
        _attn_check(ctx, c, Hq, Hkv, q, k, v)


def test_attention_equal_scores_in_long_rows():
    """Weights all equal: the sum over thousands of small values."""
    gen = _gen(17)
    c = Cache(gen, 1, (12000,), (1,))
    z = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device=DEV)
    with Ctx(4, 1) as ctx:
        _attn_check(ctx, c, 4, 1, z, z[:, :1].contiguous(), (z[:, :1] + 0.25).contiguous())


@pytest.mark.parametrize("L, S", [((70, 0, 33), (1, 3, 40)), ((5003,), (2,))])
def test_attention_equal_scores_of_any_size(L, S):
    """Keys all equal (0.5 everywhere), queries of one element, up to 2^100: every score is the same product, in the cache and in the
    suffix, and weights are even however large it is and whatever the value rows' s are."""
    gen = _gen(43)
    Hq, Hkv = 16, 2
    c = Cache(gen, Hkv, L, S)
    n = c.pages[0].shape[0] * Hkv
    page = c.pages.view(n, R.PAGE)
    page[:, :1024] = 0
    half = torch.zeros(n, 16, 2, dtype=torch.float16, device=DEV)
    half[:, :, 1] = 0.5
    page[:, 2048:2112] = half.view(n, 32).view(torch.uint8)
    par = page[:, 2112:2176].contiguous().view(torch.float16).view(n, 16, 2)
    par[:, :, 0] *= 2.0 ** torch.randint(-6, 7, (n, 16), generator=gen, device=DEV).half()
    page[:, 2112:2176] = par.view(n, 32).view(torch.uint8)
    q = torch.zeros(c.T, Hq, 128, device=DEV)
    size = [0, 5, 12, 14, 16, 18, 22, 25, 28, 31, 36, 50, 70, 100]
    for h in range(Hq):
        for t in range(c.T):
            q[t, h, (7 * t + h) % 128] = (-1.0) ** (t + h // 2) * 2.0 ** size[(3 * t + h) % len(size)]
    k = torch.full((c.T, Hkv, 128), 0.5, device=DEV).bfloat16()
    v = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    out = torch.empty(c.T, Hq * 128, dtype=torch.bfloat16, device=DEV)
    with Ctx(Hq, Hkv) as ctx:
        cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, 0, q.bfloat16(), k, v, out, c.scratch(ctx))
    for b, (l, s) in enumerate(zip(L, S)):
        ids = torch.as_tensor(c.table[b][:(l + 15) // 16].astype(np.int64), device=DEV)
        for h in range(Hkv):
            vc, vs, vz = R.read_pages(c.pages[0][ids, h])[1] if l else (torch.zeros(0, 16, 128, device=DEV).double(),) + (torch.zeros(0, 16, device=DEV).double(),) * 2
            sc = (vs[..., None] * vc).reshape(-1, 128)[:l]
            z = vz.reshape(-1)[:l, None].expand(-1, 128)
            for i in range(s):
                t = int(c.cu[b]) + i
                suffix = v[int(c.cu[b]):t + 1, h].double()
                m = l + i + 1
                want = (sc.sum(0) + z.sum(0) + suffix.sum(0)) / m
                apart = (sc.sum(0) + z.abs().sum(0) + suffix.abs().sum(0)) / m
                # half a step of the result; of p s as a half, whose smallest step is 2^-24 for p = 2^-2; scores below 2^14 are rounded
                # to 2^-11 in the suffix and not in the cache; sums
                tol = 2.0 ** -8 * want.abs() + 2.0 ** -11 * sc.sum(0) / m + 15 * 2.0 ** -23 + (2.0 ** -10 + (m / 32 + 64) * 2.0 ** -24 * 6) * apart
                got = out[t].view(Hkv, Hq // Hkv, 128)[h].double()
                assert bool(((got - want).abs() <= tol).all()), (b, h, i, float(((got - want).abs() / tol).max()))


def test_attention_a_nan_stays_in_its_head():
    gen = _gen(18)
    Hq, Hkv = 8, 2
    c = Cache(gen, Hkv, (100, 20), (2, 1))
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV).bfloat16()
    k = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    v = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    with Ctx(Hq, Hkv) as ctx:
        good = _attn_check(ctx, c, Hq, Hkv, q, k, v).view(c.T, Hq, 128)
        q[1, 2, 5] = float("nan")
        out = torch.empty(c.T, Hq * 128, dtype=torch.bfloat16, device=DEV)
        cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, 0, q, k, v, out, c.scratch(ctx))
        torch.cuda.synchronize()
    out = out.view(c.T, Hq, 128)
    assert bool(torch.isnan(out[1, 2]).all())
    keep = torch.ones(c.T, Hq, dtype=torch.bool, device=DEV)
    keep[1, 2] = False
    assert torch.equal(out[keep], good[keep])


@pytest.mark.parametrize("Hq, Hkv, S", [(4, 2, 5), (6, 1, 40), (40, 8, 33), (12, 2, 100)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_attention_what_a_later_token_holds_stays_out(Hq, Hkv, S, bad):
    """Keys and values of a suffix token that are not finite reach the rows from that token on, and no other."""
    gen = _gen(41)
    c = Cache(gen, Hkv, (50, 3), (S, 2))
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV).bfloat16()
    k = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    v = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    at = S // 2
    for name in ("v", "k"):
        kk, vv = k.clone(), v.clone()
        with Ctx(Hq, Hkv) as ctx:
            good = _attn_check(ctx, c, Hq, Hkv, q, kk, vv).view(c.T, Hq, 128)
            if name == "v":
                vv[at, Hkv - 1, 77] = bad
            else:
                kk[at, Hkv - 1, 77] = float("nan")
            out = torch.empty(c.T, Hq * 128, dtype=torch.bfloat16, device=DEV)
            cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, 0, q, kk, vv, out, c.scratch(ctx))
            torch.cuda.synchronize()
        out, G = out.view(c.T, Hq, 128), Hq // Hkv
        seen = torch.zeros(c.T, Hq, 128, dtype=torch.bool, device=DEV)
        seen[at:S, (Hkv - 1) * G:, slice(77, 78) if name == "v" else slice(None)] = True
        assert torch.equal(out[~seen], good[~seen])
        assert not bool(torch.isfinite(out[seen]).any())


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_attention_what_a_later_token_holds_stays_out_of_many_rows(bad):
    """The same where four wavefronts have 32 rows each, and chunks of keys that some of them see as a whole."""
    gen = _gen(44)
    Hq, Hkv, S = 40, 8, 100
    c = Cache(gen, Hkv, (20,) * 6, (S,) * 6)
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV).bfloat16()
    k = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    v = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    outs = []
    with Ctx(Hq, Hkv) as ctx:
        for at in (None, 2 * S + 45):
            if at is not None:
                v[at, 3, 77] = bad
            out = torch.empty(c.T, Hq, 128, dtype=torch.bfloat16, device=DEV)
            cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, 0, q, k, v, out, c.scratch(ctx))
            outs.append(out)
        torch.cuda.synchronize()
    seen = torch.zeros(c.T, Hq, 128, dtype=torch.bool, device=DEV)
    seen[2 * S + 45:3 * S, 15:20, 77] = True
    assert torch.equal(outs[1][~seen], outs[0][~seen])
    assert not bool(torch.isfinite(outs[1][seen]).any())


def test_cache_beyond_4_gib():
    """Pages whose byte offsets pass 32 bits."""
    Hq, Hkv = 4, 2
    n_blocks = 1_100_000                                # 4.8 GB
    gen = _gen(19)
    pages = torch.empty(1, n_blocks, Hkv, R.PAGE, dtype=torch.uint8, device=DEV)
    small = Cache(gen, Hkv, (70, 33), (6, 2))
    far = [int(x) for x in np.linspace(n_blocks - 1, 1_000_000, int(small.n_blocks))]
    for i, blk in enumerate(far):
        pages[0, blk] = small.pages[0, i]
    table = np.where(small.table < small.n_blocks, np.asarray(far, dtype=np.int32)[np.minimum(small.table, small.n_blocks - 1)], 0).astype(np.int32)
    dev_table = torch.from_numpy(table).to(DEV)
    kv = cb.make_kv4(pages, dev_table, n_blocks, 16, table.shape[1])
    q = torch.randn(small.T, Hq, 128, generator=gen, device=DEV).bfloat16()
    k = torch.randn(small.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    v = torch.randn(small.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    qkv = torch.randn(small.T, (Hq + 2 * Hkv) * 128, generator=gen, device=DEV)
    res = []
    with Ctx(Hq, Hkv) as ctx:
        for cache in (small.kv, kv):
            out = torch.empty(small.T, Hq * 128, dtype=torch.bfloat16, device=DEV)
            cb.confspec_op_kv4_attention(ctx, cache, small.batch, 0, q, k, v, out, small.scratch(ctx))
            qq, kk, vv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
            kr, vr = (torch.empty(small.T, Hkv, 128, device=DEV) for _ in range(2))
            cb.confspec_op_kv4_append(ctx, cache, small.batch, 0, qkv, None, None, qq, kk, vv)
            cb.confspec_op_kv4_read(ctx, cache, small.batch, 0, kr, vr)
            res.append((out, kr, vr))
    for x, y in zip(*res):
        assert torch.equal(x, y)


def test_block_ids_out_of_range_are_clamped():
    gen = _gen(20)
    Hq, Hkv = 4, 2
    c = Cache(gen, Hkv, (100, 40), (1, 2))
    c.table[0, 1], c.table[1, 0] = -5, c.n_blocks + 1000
    c.keep[0][0].copy_(torch.from_numpy(c.table))
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV).bfloat16()
    k = torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16()
    with Ctx(Hq, Hkv) as ctx:
        _attn_check(ctx, c, Hq, Hkv, q, k, k.clone())


# ---------------------------------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------------------------------
class Layer:
    """One layer of a step on 4-bit weights and cache, the way the header lists the calls."""

    def __init__(self, d, Hq, Hkv, F, group, seed):
        gen = _gen(seed)
        self.d, self.Hq, self.Hkv, self.F, self.g = d, Hq, Hkv, F, group
        self.ptr = cb.confspec_create(cb.make_model_cfg(1, d, Hq, Hkv, 128, F, 1024, THETA, 1e-6, "bf16"), 0)
        self.shapes = dict(qkv=((Hq + 2 * Hkv) * 128, d), o=(d, Hq * 128), gu=(2 * F, d), down=(d, F))
        self.w, self.packed = {}, {}
        for name, (N, K) in self.shapes.items():
            codes, s, z, self.w[name] = R.w4_quantise_case(gen, N, K, group, DEV)
            self.packed[name] = torch.empty(cb.confspec_w4_bytes(N, K, group), dtype=torch.uint8, device=DEV)
            cb.confspec_w4_pack(self.ptr, codes, s, z, N, K, group, self.packed[name], gate_up=name == "gu")
        self.g1, self.g2 = ((1 + 0.1 * torch.randn(d, generator=gen, device=DEV)).bfloat16() for _ in range(2))
        torch.cuda.synchronize()

    def buffers(self, c):
        T, d, f32, b16 = c.T, self.d, torch.float32, torch.bfloat16
        e = lambda *s, dt=f32: torch.empty(*s, dtype=dt, device=DEV)
        return dict(h=e(T, d, dt=b16), qkv=e(T, (self.Hq + 2 * self.Hkv) * 128), q=e(T, self.Hq, 128, dt=b16), k=e(T, self.Hkv, 128, dt=b16),
                    v=e(T, self.Hkv, 128, dt=b16), att=e(T, self.Hq * 128, dt=b16), act=e(T, self.F, dt=b16), y=e(T, d), scratch=c.scratch(self.ptr))

    def run(self, c, x, w, stream=None):
        p, T, g = self.ptr, c.T, self.g
        mm = lambda a, name, res, out, epi: cb.confspec_op_w4_gemm(p, a, self.packed[name], res, out, T, *self.shapes[name], g, epi, stream=stream)
        cb.confspec_op_rmsnorm(p, x, self.g1, w["h"], T, stream=stream)
        mm(w["h"], "qkv", None, w["qkv"], cb.EPI_STORE_F32)
        cb.confspec_op_kv4_append(p, c.kv, c.batch, 0, w["qkv"], None, None, w["q"], w["k"], w["v"], stream=stream)
        cb.confspec_op_kv4_attention(p, c.kv, c.batch, 0, w["q"], w["k"], w["v"], w["att"], w["scratch"], stream=stream)
        mm(w["att"], "o", x, w["y"], cb.EPI_RESID_F32)
        cb.confspec_op_rmsnorm(p, w["y"], self.g2, w["h"], T, stream=stream)
        mm(w["h"], "gu", None, w["act"], cb.EPI_SWIGLU)
        mm(w["act"], "down", w["y"], w["y"], cb.EPI_RESID_F32)
        return w["y"]

    def reference(self, c, pages, x):
        """float64, with the roundings to bf16 where the calls make them."""
        r16 = lambda t: t.float().bfloat16().double()
        norm = lambda t, g: r16(t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6) * g.double())
        x = x.double()
        qkv = (norm(x, self.g1) @ self.w["qkv"].t()).view(c.T, -1, 128)
        pos = torch.from_numpy(np.concatenate([l + np.arange(s) for l, s in zip(c.L, c.S)])).to(DEV)
        rot = r16(R.rotate(qkv[:, :self.Hq + self.Hkv], pos, THETA))
        q, k, v = rot[:, :self.Hq], rot[:, self.Hq:], r16(qkv[:, self.Hq + self.Hkv:])
        att, _ = R.attention(pages[0], c.table, q, k, v, c.cu, c.lens, self.Hq, self.Hkv)
        y = x + r16(att) @ self.w["o"].t()
        gu = norm(y, self.g2) @ self.w["gu"].t()
        gate, up = gu[:, :self.F], gu[:, self.F:]
        return y + r16(gate / (1 + torch.exp(-gate)) * up) @ self.w["down"].t()


@pytest.mark.parametrize("d, Hq, Hkv, F, group, L, S", [(512, 4, 2, 768, 128, (200, 0, 33), (1, 1, 1)), (768, 6, 1, 1280, 64, (500, 64), (3, 8)),
                                                        (1536, 12, 2, 8960, 128, (900, 1700, 5, 64), (1, 1, 1, 1)), (512, 4, 4, 512, 32, (90,), (100,))])
def test_a_layer_in_4_bits(d, Hq, Hkv, F, group, L, S):
    lay = Layer(d, Hq, Hkv, F, group, 21)
    gen = _gen(22)
    c = Cache(gen, Hkv, L, S)
    before = c.pages.clone()
    x = torch.randn(c.T, d, generator=gen, device=DEV)
    y = lay.run(c, x, lay.buffers(c))
    torch.cuda.synchronize()
    ref = lay.reference(c, before, x)
    # x + two branches; every 16-bit rounding on the way (norm, q / k / v, attention, activation) is 2^-8 of what it rounds at
    # most and spreads over a projection's sum: the branch's error stays within 4 such roundings of its size (rms over a row)
    err = (y.double() - ref).pow(2).mean(-1).sqrt()
    size = (ref - x.double()).pow(2).mean(-1).sqrt()
    print(f"layer {d}: error {float((err / size).max()):.2e} of the branches", flush=True)
    assert bool((err <= 4 * 2.0 ** -8 * size).all())
    cb.confspec_destroy(lay.ptr)


def test_a_layer_on_two_streams_and_in_two_graphs():
    """Eager on two streams, then captured, each with buffers of its own; replays between eager calls give what the eager
    calls gave.  The second step of a trace reads the rows that the first one appended."""
    lay = Layer(512, 4, 2, 768, 64, 23)
    caches, xs, bufs, want, pages0 = [], [], [], [], []
    for i, (L, S) in enumerate((((300, 17, 2000), (1, 1, 1)), ((40, 700), (6, 11)))):
        gen = _gen(24 + i)
        c = Cache(gen, 2, L, S)
        caches.append(c)
        pages0.append(c.pages.clone())
        xs.append(torch.randn(c.T, 512, generator=gen, device=DEV))
        bufs.append(lay.buffers(c))
        want.append(lay.run(c, xs[i], bufs[i]).clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, s in enumerate(streams):
        bufs[i]["y"].zero_()
        caches[i].pages.copy_(pages0[i])
    torch.cuda.synchronize()
    for i, s in enumerate(streams):
        lay.run(caches[i], xs[i], bufs[i], stream=s)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(bufs[i]["y"], want[i])
    graphs = []
    for i, s in enumerate(streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            lay.run(caches[i], xs[i], bufs[i])
        graphs.append(g)
    for rep in range(4):
        for i in range(2):
            caches[i].pages.copy_(pages0[i])
            for name in ("y", "qkv", "att", "act"):
                bufs[i][name].fill_(float("nan"))
            if rep % 2:
                bufs[i]["scratch"].fill_(255)
        torch.cuda.synchronize()
        for i in (0, 1) if rep % 2 else (1, 0):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(bufs[i]["y"], want[i]), (rep, i)
        other = Cache(_gen(30 + rep), 2, (100,), (2,))
        lay.run(other, xs[0][:2].contiguous(), lay.buffers(other))
        torch.cuda.synchronize()
    cb.confspec_destroy(lay.ptr)


def test_tokens_one_at_a_time_see_the_rows_appended():
    """Decoding: step n attends over the rows that the steps before stored.  Against a cache that the plain form quantised."""
    Hq, Hkv, steps = 6, 2, 20
    gen = _gen(40)
    L0 = (13, 0, 47)
    c0 = Cache(gen, Hkv, L0, (steps,) * 3)
    qkv = torch.randn(steps, 3, (Hq + 2 * Hkv) * 128, generator=gen, device=DEV)
    plain = c0.pages.cpu().clone()
    with Ctx(Hq, Hkv) as ctx:
        for n in range(steps):
            lens = np.asarray(L0, dtype=np.int32) + n
            dl, cu = torch.from_numpy(lens).to(DEV), np.arange(4, dtype=np.int32)
            dcu = torch.from_numpy(cu).to(DEV)
            batch, keep = cb.make_batch(c0.ids, dcu, dl, cu, lens)
            q = torch.empty(3, Hq, 128, dtype=torch.bfloat16, device=DEV)
            k, v = (torch.empty(3, Hkv, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            out = torch.empty(3, Hq * 128, dtype=torch.bfloat16, device=DEV)
            need = cb.confspec_op_kv4_attention_scratch_bytes(ctx, batch)
            scratch = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
            cb.confspec_op_kv4_append(ctx, c0.kv, batch, 0, qkv[n], None, None, q, k, v)
            cb.confspec_op_kv4_attention(ctx, c0.kv, batch, 0, q, k, v, out, scratch)
            torch.cuda.synchronize()
            ref, tol = R.attention(plain[0].to(DEV), c0.table, q, k, v, cu, lens, Hq, Hkv)
            assert bool(((out.double() - ref).abs() <= tol).all()), n
            for name, x in (("k", k), ("v", v)):
                cc, ss, zz = (y.cpu() for y in R.quantise(x))
                for b in range(3):
                    for h in range(Hkv):
                        R.write_row(plain[0], int(c0.table[b, lens[b] // 16]), h, int(lens[b]) % 16, cc[b, h], ss[b, h], zz[b, h], name == "v")
    assert torch.equal(plain, c0.pages.cpu())
