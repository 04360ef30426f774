"""Products with 4-bit weights and the 4-bit paged cache on values at the ends of their types, and at the ends of their
buffers; formats and bounds of tests/int4_ref.py."""
import numpy as np
import pytest
import torch

from paper_2602_18447_amd import binding as cb
from tests import int4_ref as R
from tests.test_gpu_int4 import DEV, Cache, Ctx, _append_case, _attn_check, _gen

pytestmark = pytest.mark.gpu
NAN_HALF = torch.tensor([0x7E00], dtype=torch.int16).view(torch.float16)[0]


# ---------------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("Hq, Hkv, L, S, n", [(4, 2, (13, 0), (12, 9), None), (1, 1, (5,), (12,), (10,)), (12, 3, (40, 7, 0), (1, 12, 30), (1, 11, 30))])
def test_append_a_row_with_a_nan_is_stored_as_nan(Hq, Hkv, L, S, n):
    """s and z are 0x7E00 and every code 0: the row reads back as NaN.  The other rows are what they are without it."""
    gen = _gen(50)
    c = Cache(gen, Hkv, L, S)
    x = torch.randn(c.T, Hq + 2 * Hkv, 128, generator=gen, device=DEV)
    nan, inf = float("nan"), float("inf")
    other = torch.tensor([-0x3FFFFF], dtype=torch.int32).view(torch.float32).item()             # with a sign and a payload
    k, v = x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    bad_k = torch.zeros(c.T, Hkv, dtype=torch.bool)
    bad_v = torch.zeros(c.T, Hkv, dtype=torch.bool)
    for bad, rows, t, h, at, value in ((bad_v, v, 1, 0, 7, nan), (bad_v, v, 3, Hkv - 1, 127, other), (bad_v, v, 4, 0, slice(None), nan), (bad_k, k, 2, 0, 3, nan),
                                       (bad_k, k, 4, Hkv - 1, 64, other), (bad_k, k, 5, 0, slice(None), nan), (bad_v, v, 10, 0, 0, nan), (bad_k, k, 11, Hkv - 1, 90, nan)):
        rows[t, h, at] = value
        bad[t, h] = True
    v[7, 0, 5], v[7, 0, 6], v[8, 0, 9] = inf, nan, -inf
    bad_v[7, 0] = True
    q, kk, vv = (torch.empty(c.T, h, 128, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))
    kr, vr = (torch.empty(c.T, Hkv, 128, device=DEV) for _ in range(2))
    want = c.pages[0].cpu()
    hn = None if n is None else np.asarray(n, dtype=np.int32)
    dn = None if n is None else torch.from_numpy(hn).to(DEV)
    with Ctx(Hq, Hkv) as ctx:
        cb.confspec_op_kv4_append(ctx, c.kv, c.batch, 0, x, dn, hn, q, kk, vv, qkv_stride=(Hq + 2 * Hkv) * 128)
        cb.confspec_op_kv4_read(ctx, c.kv, c.batch, 0, kr, vr)
        torch.cuda.synchronize()
    assert torch.equal(torch.isnan(kk).any(-1).cpu(), bad_k) and torch.equal(torch.isnan(vv).any(-1).cpu(), bad_v)
    none = torch.zeros(128, dtype=torch.int64)
    for rows, bad, got, is_v in ((kk.cpu(), bad_k, kr.cpu(), False), (vv.cpu(), bad_v, vr.cpu(), True)):
        cc, ss, zz = R.quantise(torch.where(bad[..., None], torch.zeros_like(rows), rows))
        for b in range(len(L)):
            for i in range(S[b] if n is None else n[b]):
                t, row = int(c.cu[b]) + i, L[b] + i
                for h in range(Hkv):
                    stored = (none, NAN_HALF, NAN_HALF) if bad[t, h] else (cc[t, h], ss[t, h], zz[t, h])
                    R.write_row(want, int(c.table[b, row // 16]), h, row % 16, *stored, is_v)
                    assert bool(torch.isnan(got[t, h]).all()) if bad[t, h] else bool(torch.isfinite(got[t, h]).all()), (b, i, h)
    assert torch.equal(want, c.pages[0].cpu())


@pytest.mark.parametrize("L, S", [((40,), (1,)), ((40, 100), (3, 1)), ((5003, 60), (2, 40)), ((20,) * 6, (100,) * 6)])
@pytest.mark.parametrize("is_v", [False, True])
def test_attention_over_a_row_stored_as_nan(L, S, is_v):
    """Every row of its trace and head is NaN, and no other."""
    gen = _gen(51)
    Hq, Hkv, j = 40, 8, 19
    c = Cache(gen, Hkv, L, S)
    q = torch.randn(c.T, Hq, 128, generator=gen, device=DEV).bfloat16()
    k, v = (torch.randn(c.T, Hkv, 128, generator=gen, device=DEV).bfloat16() for _ in range(2))
    with Ctx(Hq, Hkv) as ctx:
        good = _attn_check(ctx, c, Hq, Hkv, q, k, v).view(c.T, Hq, 128)
        none = torch.zeros(128, dtype=torch.int64, device=DEV)
        R.write_row(c.pages[0], int(c.table[0, j // 16]), 3, j % 16, none, NAN_HALF.to(DEV), NAN_HALF.to(DEV), is_v)
        out = torch.empty(c.T, Hq, 128, dtype=torch.bfloat16, device=DEV)
        cb.confspec_op_kv4_attention(ctx, c.kv, c.batch, 0, q, k, v, out, c.scratch(ctx))
        torch.cuda.synchronize()
    seen = torch.zeros(c.T, Hq, dtype=torch.bool, device=DEV)
    seen[:S[0], 15:20] = True
    assert bool(torch.isnan(out[seen]).all()) and torch.equal(out[~seen], good[~seen])


def test_append_a_zero_has_no_sign():
    """Rows whose minimum or range rounds to a zero half from below: bytes as the plain form has them."""
    def edit(x, Hq, Hkv):
        for rows in (x[:, Hq + Hkv:], x[:1, Hq:Hq + Hkv]):             # (keys at position 0 are not turned)
            for t in range(rows.shape[0]):
                rows[t] = torch.rand(Hkv, 128, generator=_gen(t), device=DEV) * 1e-3
        v = x[:, Hq + Hkv:]
        v[0, :, 3] = -1e-9                                             # z from (-2^-25, 0)
        v[1, :, 100] = -2.0 ** -26
        v[2] = 1.5 * 2.0 ** -25                                        # z is 2^-24, beyond the maximum: s from below 0
        v[3] = -2.0 ** -26
        v[4] = -0.0
        v[5] = -1e-9
        v[5, :, 9] = 1e-9
        x[0, Hq:Hq + Hkv, 70] = -1e-9
    _append_case(3, 3, (0,), (6,), None, 52, edit=edit)
