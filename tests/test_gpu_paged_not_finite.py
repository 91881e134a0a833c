"""ss_paged_attention of rows whose scores are no numbers: NaN comes out, and only where such a score was seen."""
import pytest
import torch

import paper_2311_04951_amd as sv
from paged_util import Cache, attention64, check_attention

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
# one launch | two: a workgroup to a head, equal parts that end inside heads; (lengths, query heads over two key heads, new rows, bound)
FORMS = {"one launch": ([0, 37, 250], 2, 1, 251), "one launch, shared": ([0, 37, 240], 8, 4, 244), "joined": ([0, 37, 900], 2, 1, 0), "joined, shared": ([0, 37, 3000], 8, 4, 0),
         "joined, many rows": ([0, 37, 700], 10, 5, 0), "one launch, many rows": ([0, 37, 100], 10, 5, 105)}


def setup(seed, dtype, form):
    lengths, heads, M, bound = FORMS[form]
    c = Cache(seed, dtype, len(lengths), 2, 64, 16, lengths, room=M)
    q = torch.randn((len(lengths), M, heads, 64), generator=c.generator).mul_(1.5).to(c.dtype)
    return c, q, bound


def attend(c, q, bound, weights):
    kv = c.device()
    w = torch.zeros(c.weight.shape, device="cuda") if weights else None
    return sv.ss_paged_attention(kv, 0, q.cuda(), weight_out=w, max_len=bound).cpu(), w.cpu() if weights else None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("form", FORMS)
def test_a_query_of_nan(dtype, weights, form):
    """One element of one row: that row alone is NaN, whatever it sees (one position, some, all pieces of a long head)."""
    c, q, bound = setup(1, dtype, form)
    clean, _ = attend(c, q, bound, weights)
    for b in range(q.shape[0]):
        for m in {0, q.shape[1] - 1}:
            for h in (0, q.shape[2] - 1):
                dirty = q.clone()
                dirty[b, m, h, 5] = NAN
                out, w = attend(c, dirty, bound, weights)
                assert out[b, m, h].isnan().all()
                rest = torch.ones(q.shape[:3], dtype=torch.bool)
                rest[b, m, h] = False
                assert torch.equal(out[rest], clean[rest])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("form", ["one launch", "joined"])
def test_keys_of_nan(dtype, weights, form):
    """All that a row sees: its own first position; a whole sequence; NaN beside scores of minus infinity.  Nothing but minus infinity: zero."""
    c, q, bound = setup(2, dtype, form)
    q[..., 0] = q[..., 0].abs() + 0.5
    n = c.lengths
    at = lambda b, s: (0, c.table[b, s // 16].long(), slice(None), s % 16)
    c.k[at(0, torch.tensor([0]))] = NAN
    c.k[at(1, torch.arange(n[1] + 1))] = NAN
    c.k[at(2, torch.arange(n[2] + 1))] = 1.0
    lowest = (0, c.table[2, torch.arange(n[2] + 1) // 16].long(), slice(None), torch.arange(n[2] + 1) % 16, 0)
    c.k[lowest] = -INF                                   # scores of sequence 2: all minus infinity
    out, _ = attend(c, q, bound, weights)
    assert out[0].isnan().all() and out[1].isnan().all() and (out[2] == 0).all()
    c.k[at(2, torch.tensor([n[2] // 2]))] = NAN          # ... but one
    out, _ = attend(c, q, bound, weights)
    assert out.isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", ["one launch, shared", "joined, shared", "one launch, many rows", "joined, many rows"])
@pytest.mark.parametrize("m", [0, 2])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_a_row_of_nan_gives_nothing_to_what_it_does_not_see(dtype, form, m, bad):
    """The newest positions, hidden from row m, hold what the rows behind it gave them; the others of its key head NaN; other heads' are as ever."""
    c, q, bound = setup(3, dtype, form)
    c.k[..., 5] = c.k[..., 5].abs() + 0.5                # (all scores of an infinite query are plus infinity)
    M, last = q.shape[1], q.shape[2] - 1
    _, gave, _ = attention64(c, 0, q, M)
    q[:, m, last, 5] = bad
    _, w = attend(c, q, bound, True)
    for (b, h), (got, off) in gave.items():
        s = torch.arange(len(got))
        at = (0, c.table[b, s // 16].long(), h, s % 16)
        have, want = w[at].double(), c.weight[at].double() + got
        hidden = len(got) - M + m + 1 if h == 1 else 0       # the first slot that row m does not see
        assert have[:hidden].isnan().all()
        assert ((have - want).abs() <= off + want * 2.0 ** -23)[hidden:].all()


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("form", ["one launch", "joined"])
def test_equal_scores_of_any_size(weights, form):
    """All scores of a row equal, from 2^20 to 2^100 either way: the mean of the values, and equal weights."""
    c, q, bound = setup(4, "f32", form)
    for power in range(20, 101):
        for sign in (1.0, -1.0):
            q[:] = 1.37 * 2.0 ** (power - 20)
            c.k[:] = sign * 1.13 * 2.0 ** 17             # 64 products times 1/8
            out, w = attend(c, q, bound, weights)
            for b, n in enumerate(c.lengths):
                s = torch.arange(n + 1)
                for h in range(2):
                    mean = c.rows(c.v, 0, b, h, n + 1).double().mean(0)
                    # values are at most 5; as many additions as there are positions
                    assert ((out[b, 0, h].double() - mean).abs() <= (n + 64) * 2.0 ** -24 * 5).all(), (power, sign, b, h)
                    if weights:
                        at = (0, c.table[b, s // 16].long(), h, s % 16)
                        want = c.weight[at].double() + 1 / (n + 1)
                        assert ((w[at].double() - want).abs() <= want * (n + 64) * 2.0 ** -24).all(), (power, sign, b, h)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("form", ["one launch, shared", "joined, shared"])
@pytest.mark.parametrize("scale,size", [(0.0, 1.0), (0.0, 1e18), (-0.0, 1e18), (1e-36, 1e18), (-3e-34, 1e17)])
def test_scales_next_to_zero(weights, form, scale, size):
    """Of products up to 1e37 a scale of zero makes equal weights, one of 1e-36 those of the definition."""
    c, q, bound = setup(5, "f32", form)
    c.k *= size
    q *= size
    kv = c.device()
    w = torch.full(c.weight.shape, 0.5, device="cuda") if weights else None
    before = w.cpu().clone() if weights else None
    out = sv.ss_paged_attention(kv, 0, q.cuda(), scale=scale, weight_out=w, max_len=bound)
    check_attention(c, 0, q, q.shape[1], out, scale, w, before)
