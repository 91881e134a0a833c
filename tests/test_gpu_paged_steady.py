"""ss_paged_attention where a wavefront goes through its ring many times and a workgroup through several heads: what long and many sequences use.

In the first test every weight is 0 or the same and every sum a whole number that 32 bits hold, so a position that is missed, read twice or in part, or
from another step of the ring changes the result by more than its rounding."""
import pytest
import torch

import paper_2311_04951_amd as sv
from paged_util import TYPES

pytestmark = pytest.mark.gpu

KV_HEADS, PAGE = 8, 32
# lengths in blocks (256 positions in bf16, 128 in fp32), the new rows among them; 0: an idle place
BLOCKS = (61.3, 0, 0.01, 3.0, 40.5, 1.0, 33.9, 17.02, 0.6, 50.0, 29.4, 12.8)
# query heads to a key head, new rows: one tile of 16 query rows, one in part, two of them, three blocks of two tiles of which the last is empty
ROWS = {"1 row": (1, 1), "9 rows": (1, 9), "24 rows": (8, 3), "80 rows": (5, 16)}


class Pages:
    def __init__(self, dtype, hd, G, M):
        T, self.hd, self.G, self.M = TYPES[dtype], hd, G, M
        self.block = 256 if dtype == "bf16" else 128
        self.n = [max(M, int(t * self.block)) if t else 0 for t in BLOCKS]
        pages = [-(-n // PAGE) for n in self.n]
        g = torch.Generator().manual_seed(hd + G)
        self.P = sum(pages) + 1
        order, self.table = torch.randperm(self.P, generator=g).to(torch.int32), torch.full((len(pages), max(pages)), -1, dtype=torch.int32)
        at = 0
        for b, count in enumerate(pages):
            self.table[b, :count] = order[at:at + count]
            at += count
        shape = (1, self.P, KV_HEADS, PAGE)
        self.k, self.v = (torch.zeros(shape + (hd,), dtype=T, device="cuda") for _ in range(2))
        self.weight = torch.zeros(shape, device="cuda")
        length = torch.tensor([n - M if n else -1 for n in self.n], dtype=torch.int32).cuda()
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.kv = sv.PagedKV(self.k, self.v, self.table.cuda(), length, weight=self.weight, position=torch.zeros(shape, dtype=torch.int32, device="cuda"),
                             status=self.status)
        self.generator = torch.Generator(device="cuda")
        self.generator.manual_seed(hd + G)

    def of(self, pool, b):
        """The positions of a sequence: [kv heads, n, ...]"""
        s = torch.arange(self.n[b])
        ids, at = self.table[b, s // PAGE].long().cuda(), (s % PAGE).cuda()
        return pool[0, ids, :, at].transpose(0, 1)

    def attend(self, q, weights, scale=None):
        out_w = torch.zeros_like(self.weight) if weights else None
        out = sv.ss_paged_attention(self.kv, 0, q, weight_out=out_w, scale=scale, max_len=max(self.n))
        assert int(self.status[0]) == 0
        return out, out_w

    def check_plan(self):
        """How many blocks of positions a workgroup has in a row, from the size of the partials; the ring's stages; pieces of several heads."""
        GM, blocks = self.G * self.M, [max(1, -(-n // self.block)) for n in self.n]
        rowblocks, row_tiles = -(-GM // 32), 1 if GM <= 16 else 2
        parts = (sv.ss_paged_attention_workspace_bytes(self.kv, KV_HEADS * self.G, self.M, max(self.n)) - 256) // (8 + 4 * self.hd)
        workgroups, stages = parts // (rowblocks * 32 * row_tiles), 128 // self.hd
        share = -(-KV_HEADS * sum(blocks) // workgroups)
        assert share >= stages + 4                             # the ring goes round, with what the first steps do not have in flight
        assert max(blocks) > share > 2 * min(blocks)           # heads of several workgroups, workgroups of several heads


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("weights", [False, True])
def test_whole_numbers(dtype, hd, rows, weights):
    G, M = ROWS[rows]
    c = Pages(dtype, hd, G, M)
    c.check_plan()
    # a key counts if its elements sum to zero (1 and -1 or -1 and 1, two at a time), not if all of them are -1
    def flip(*shape, p=0.5):
        return torch.rand(shape, generator=c.generator, device="cuda") < p
    counts = flip(*c.k.shape[:-1])
    pairs = torch.where(flip(*c.k.shape[:-1], hd // 2), 1.0, -1.0)
    c.k.copy_(torch.where(counts[..., None], torch.stack([pairs, -pairs], -1).flatten(-2), -1.0))
    c.v.copy_(torch.where(flip(*c.v.shape), 1.0, -1.0) * flip(*c.v.shape, p=0.06))
    q = torch.ones((len(c.n), M, KV_HEADS * G, hd), dtype=c.k.dtype, device="cuda")
    out, w = c.attend(q, weights, scale=8.0)                   # scores 0 and -8 hd: exp2 of that is 0
    half_step = torch.finfo(out.dtype).eps / 2
    expected_w = torch.zeros_like(c.weight, dtype=torch.float64)
    for b, n in enumerate(c.n):
        if n == 0:
            assert not out[b].any()
            continue
        counted, v = c.of(counts, b), c.of(c.v, b).double()
        got = torch.zeros(counted.shape, dtype=torch.float64, device="cuda")
        for m in range(M):
            see = n - M + m + 1
            seen = counted[:, :see] | ~counted[:, :see].any(1, keepdim=True)   # (if none counts, all of them do)
            count = seen.sum(1, keepdim=True).double()
            total = (v[:, :see] * seen[:, :, None]).sum(1)
            assert total.abs().max() * half_step < 0.5                        # one more or less is more than the rounding
            want = (total / count)[:, None]
            error = (out[b, m].double().reshape(KV_HEADS, G, hd) - want).abs()
            assert (error <= want.abs() * (half_step + 2.0 ** -22)).all(), (b, m)
            got[:, :see] += G * seen / count
        s = torch.arange(n)
        ids, at = c.table[b, s // PAGE].long().cuda(), (s % PAGE).cuda()
        expected_w[0, ids, :, at] = got.T
    if weights:
        assert ((w.double() - expected_w).abs() <= expected_w * (G * M + 8) * 2.0 ** -24).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("rows", ROWS)
def test_any_numbers(dtype, hd, rows):
    """Against 64 bits, two key heads of every sequence, and the same bits again."""
    G, M = ROWS[rows]
    c = Pages(dtype, hd, G, M)
    for pool in (c.k, c.v):
        pool.normal_(generator=c.generator)
    q = torch.randn((len(c.n), M, KV_HEADS * G, hd), generator=c.generator, device="cuda").mul_(1.5).to(c.k.dtype)
    out, w = c.attend(q, True)
    again, w_again = c.attend(q, True)
    assert torch.equal(out, again) and torch.equal(w, w_again)
    half_step = torch.finfo(out.dtype).eps / 2
    for b, n in enumerate(c.n):
        if n == 0:
            continue
        k, v, have = c.of(c.k, b), c.of(c.v, b), c.of(w, b)
        see = torch.arange(n, device="cuda") <= torch.arange(n - M, n, device="cuda").repeat(G)[:, None]
        for h in (b % KV_HEADS, KV_HEADS - 1):
            x = q[b, :, h * G:(h + 1) * G].transpose(0, 1).reshape(G * M, hd).double()
            kd, vd = k[h].double(), v[h].double()
            p = torch.softmax((x @ kd.T / hd ** 0.5).masked_fill(~see, float("-inf")), -1)
            want = p @ vd
            # as in paged_util.attention64: scores' products and scaling, weights of 16 bits, additions
            score = (hd + 4) * 2.0 ** -24 * ((x.abs() @ kd.abs().T / hd ** 0.5).max(1).values + 1)
            rel = 2 * score + (2.0 ** -17 if dtype == "bf16" else 0) + (n / 16 + 64) * 2.0 ** -24
            bound = rel[:, None] * (p @ vd.abs())
            got = out[b, :, h * G:(h + 1) * G].transpose(0, 1).reshape(G * M, hd).double()
            assert ((got - want).abs() <= bound + half_step * (want.abs() + bound)).all(), (b, h)
            sums = p.sum(0)
            assert ((have[h].double() - sums).abs() <= (p * rel[:, None]).sum(0) + sums * 2.0 ** -23).all(), (b, h)
