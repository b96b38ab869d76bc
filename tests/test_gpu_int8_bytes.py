"""Int8 attention: a row's bytes where its value reference is at the point of rising, and weights far below a row's largest."""

import numpy as np
import pytest
import torch

from oracle import int8 as oracle
from tests.packed_helpers import host
from tests.test_gpu_packed import bits, kvg  # noqa: F401

pytestmark = pytest.mark.gpu

CTX, HKV = 95, 16                     # the first row sees three blocks of 32 keys
KEY_SCALES = (3.0, 7.0, 70.0, 700.0)  # a layer's


class Crossing:
    """Two query heads a KV head.  The first one's scores are equal over two blocks of keys, s; the second block's values have the
    scale at which log2 of the largest weighted value, s + log2(scale), meets the least one that raises the row's reference, from one
    half of a last bit below to two above over the KV heads.  The third block's keys weigh 2^-8 to 2^-30 of the others' and alone have values
    in the first 32 dimensions, one each: their roundings show in the result.  The other head may raise its own reference in the
    second block or not."""

    def __init__(self, kvg, D, room):  # noqa: F811
        L, pages = len(KEY_SCALES), 9
        max_pages = -(-(room + 40) // 16)
        table = np.zeros((1, max_pages), dtype=np.int32)
        table[0, :pages] = np.random.default_rng(3).permutation(pages)
        k, v = (np.zeros((L, pages * 16, HKV, D), dtype=np.int8) for _ in range(2))
        k[:, :96, :, 0] = 100
        k[:, 64:96, :, 1] = -(30 + np.arange(32))[None, :, None]
        k[:, :32, :, 2] = 127
        k[:, 32:64, :, 3] = 127
        rng = np.random.default_rng(5)
        v[:, :64, :, 32:] = rng.integers(-127, 128, (L, 64, HKV, D - 32))
        for j in range(32):
            v[:, 64 + j, :, j] = 127
        ks = np.repeat(np.float32(KEY_SCALES)[:, None, None], pages, axis=1) * np.ones((1, 1, HKV), dtype=np.float32)
        vs = np.ones((L, pages, HKV), dtype=np.float32)
        self.q = np.zeros((L, 1, 2, D), dtype=np.float32)
        for l, sk in enumerate(np.float32(KEY_SCALES)):
            log2e = np.float32(1.4426950408889634)
            kq = np.float32(2.0 ** -13) * log2e * sk
            s = np.float32(819200.0) * kq                              # of 100 in the first dimension, in log2 units
            m = np.ceil(s / 16) * 16
            meet = np.ceil(s - m) + 8 + m                              # the first block's reference, raised by eight
            half_bit = float(np.spacing(np.float32(meet))) / 2
            off = half_bit * (np.arange(HKV) / (HKV - 1) * 3 - 1)
            vs[l, 2:4] = np.exp2(meet - float(s) + off)
            # an integer of the second dimension is a quarter to half a unit of the score
            self.q[l, 0, 0, :2] = 1.0, 2.0 ** np.floor(np.log2(0.5 / (float(log2e) * float(sk))))
        slots = torch.from_numpy(table[0, :pages].astype(np.int64)).cuda()
        self.kvg, self.D = kvg, D
        self.cache = kvg.Int8Cache.allocate(L, pages, 2 * HKV, HKV, D)
        for pool, x in ((self.cache.k_pool, k), (self.cache.v_pool, v)):
            pool[:, slots] = torch.from_numpy(x.reshape(L, pages, 16, HKV, D).transpose(0, 1, 3, 2, 4).copy()).cuda()
        for scale, x in ((self.cache.k_scale, ks), (self.cache.v_scale, vs)):
            scale[:, slots] = torch.from_numpy(x).cuda()
        self.seqs = kvg.Seqs(torch.from_numpy(table).cuda(), torch.tensor([CTX], dtype=torch.int32, device="cuda"),
                             torch.zeros(1, dtype=torch.int64, device="cuda"), room)

    def attend(self, n, raising):
        """n rows, of which the ones in `raising` have a second head that raises its reference in the second block: the first head's
        result, bits [L][n][HKV][D]."""
        kvg, L = self.kvg, len(KEY_SCALES)  # noqa: F811
        q = np.repeat(np.repeat(self.q, n, axis=1)[:, :, None], HKV, axis=2)       # [L][n][HKV][2][D]
        q[:, :, :, 1, 2] = 1.0
        for t in raising:
            q[:, t, :, 1, 2:4] = 0.0, 1.0
        q = torch.from_numpy(q.reshape(L, n, 2 * HKV, self.D)).cuda().to(torch.bfloat16)
        packed = kvg.Packed(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, n)
        out = torch.empty_like(q)
        kvg.kvg_int8_attn(self.cache, self.seqs, packed, 0, L, q, 1.0, out, kvg.int8_attn_workspace(self.cache, self.seqs, packed, L))
        assert bool(out.isfinite().all())
        return bits(out.view(L, n, HKV, 2, self.D)[:, :, :, 0].contiguous())


@pytest.mark.parametrize("D", [64, 128, 256])
def test_a_row_at_its_references_rise(kvg, D):  # noqa: F811
    """The same bytes beside heads and rows that raise their references and beside ones that do not, in single tokens, short chunks and
    tiles, of one segment and split."""
    want = None
    for room in (CTX, 2600):
        c = Crossing(kvg, D, room)
        for n, raising in ((1, ()), (1, (0,)), (16, ()), (16, (9,)), (40, ()), (40, (5,)), (40, (20, 39)), (40, range(40))):
            got = c.attend(n, raising)
            if want is None:
                want = got
            # every row has the first one's query, and the tokens between weigh nothing
            wrong = (got != want).any(dim=3).nonzero()
            assert len(wrong) == 0, f"room {room}, {n} rows, raising {list(raising)}: (layer, row, KV head) {wrong[:8].tolist()} of {len(wrong)}"


@pytest.mark.parametrize("heads", [(2, 2, 64), (4, 2, 128), (8, 4, 256)])
@pytest.mark.parametrize("n", [1, 40])
def test_weights_far_below_the_largest(kvg, heads, n):  # noqa: F811
    """Equal scores, one page of values of scale 1 and the others of 2^-18 to 2^-20: the former has no values in half of the dimensions, where
    the result is that of the light pages.  Their scales lie between fp16's steps for a largest weight of 1 or less, by 1/32 of themselves."""
    Hq, Hkv, D = heads
    rng = np.random.default_rng(8)
    pages, ctx = 24, 16 * 24 - n
    kn, vn = rng.integers(-127, 128, (pages * 16, Hkv, D)), rng.integers(64, 128, (pages * 16, Hkv, D))
    vn[:16, :, D // 2:] = 0
    vs = np.tile((1 + 3 / 32) * np.exp2(-20.0 + np.arange(Hkv) % 3), (pages, 1))
    vs[0] = 1.0
    ks = np.ones((pages, Hkv))
    cache = kvg.Int8Cache.allocate(1, pages, *heads)
    for pool, x in ((cache.k_pool, kn), (cache.v_pool, vn)):
        pool[0].copy_(torch.from_numpy(x.reshape(pages, 16, Hkv, D).transpose(0, 2, 1, 3).astype(np.int8)))
    for scale, x in ((cache.k_scale, ks), (cache.v_scale, vs)):
        scale[0].copy_(torch.from_numpy(x))
    seqs = kvg.Seqs(torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous(), torch.tensor([ctx], dtype=torch.int32, device="cuda"),
                    torch.zeros(1, dtype=torch.int64, device="cuda"), ctx)
    packed = kvg.Packed(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, n)
    q = torch.zeros(1, n, Hq, D, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    kvg.kvg_int8_attn(cache, seqs, packed, 0, 1, q, 0.1, out, kvg.int8_attn_workspace(cache, seqs, packed, 1))
    want, tol = oracle.attend(host(q[0]), ctx + np.arange(n), kn, np.repeat(ks, 16, axis=0), vn, np.repeat(vs, 16, axis=0), 0.1)
    assert np.all(np.abs(host(out[0]) - want) <= tol)
