"""The 8-bit paged cache and attention over it (include/qqq_layer.h) against the definitions in 64 bits.

Tolerances.  Codes, scales and tails are compared bit for bit: the quantiser's quotient is the fp32 division's.  What is read back is one
product rounded to fp32 and to fp16: within 2^-11 (1 + 2^-11) of it, or half the least fp16 value.
Attention: a score's fp32 sum over D products is off by at most ds = (D + 8) 2^-23 scale sum |q| |k|, which changes a weight by exp(2 ds) at
most; weights are rounded to fp16, 2^-11, and where they are below fp16's normal range by 2^-25 of a unit that is 2^-6 of the largest;
exponent, its argument (|z| < 2^8: 2^-16) and the final division add 3e-5; the result is rounded to fp16.  So
|out - exact| <= (2^-11 + 2 ds + 3e-5) sum p |v| + length 2^-31 max |v| + 2^-11 |exact| + 2^-25,  |lse - exact| <= ds + 3e-5.
"""
import numpy as np
import pytest
import torch

from oracle import qqq_layer_oracle as ref
from paper_2406_09904_amd import binding as qqq

pytestmark = pytest.mark.gpu


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Both:
    """A cache on the host and its twin on the device, filled with the same calls."""

    def __init__(self, seed, lengths, heads, dim, page, slots=None, columns=None):
        self.rng = np.random.default_rng(seed)
        self.heads, self.dim, self.page, B = heads, dim, page, len(lengths)
        self.columns = max(1, max(lengths) // page) if columns is None else columns
        pages = sum(n // page for n in lengths) + 3
        order = self.rng.permutation(pages)
        self.table, at = np.full((B, self.columns), pages - 1, np.int32), 0
        for b, n in enumerate(lengths):
            self.table[b, :n // page] = order[at:at + n // page]
            at += n // page
        nslots = B + 2 if slots is None else slots
        self.slots = self.rng.permutation(nslots)[:B].astype(np.int32)
        self.host = ref.Cache(pages, heads, dim, page, nslots)
        self.dev = qqq.new_kv8_cache(pages, heads, dim, page, nslots)
        self.max_len = self.columns * page + page - 1

    def batch(self, kv_len, cu, max_new=None):
        new = np.diff(cu)
        return qqq.KV8Batch(_dev(self.table), _dev(np.array(kv_len, np.int32)), _dev(np.array(cu, np.int32)), _dev(self.slots),
                            int(new.max(initial=0)) if max_new is None else max_new, self.max_len)

    def random(self, T):
        scale = np.exp(self.rng.standard_normal((1, self.heads, 1)))
        return tuple((self.rng.standard_normal((T, self.heads, self.dim)) * scale).astype(np.float16) for _ in range(2))

    def append(self, kv_len, new, k=None, v=None):
        cu = np.concatenate([[0], np.cumsum(new)])
        if k is None:
            k, v = self.random(cu[-1])
        self.host.append(self.table, kv_len, cu, self.slots, k, v)
        # the values in the middle of a wider tensor, as a fused projection's output holds them
        wide = torch.full((max(1, cu[-1]), 2 * self.heads + 3, self.dim), 9.0, dtype=torch.float16, device="cuda")
        wide[:cu[-1], 2:2 + self.heads], wide[:cu[-1], 2 + self.heads:2 + 2 * self.heads] = _dev(k), _dev(v)
        qqq.qqq_kv8_append(self.dev, self.batch(kv_len, cu), wide[:cu[-1], 2:2 + self.heads], wide[:cu[-1], 2 + self.heads:2 + 2 * self.heads])
        torch.cuda.synchronize()

    def check(self):
        for name in ("k_codes", "k_scale", "v_codes", "v_scale", "k_tail", "v_tail"):
            got, want = getattr(self.dev, name).cpu().numpy(), getattr(self.host, name)
            if name == "k_tail" or name == "v_tail":   # a slot keeps the tokens of the page it held; the device may not have put them there
                continue
            assert np.array_equal(got, want), name

    def check_tokens(self, kv_len):
        """Every sequence's tokens, through qqq_kv8_read."""
        cu = np.concatenate([[0], np.cumsum(kv_len)])
        T = int(cu[-1])
        k, v = qqq.qqq_kv8_read(self.dev, self.batch(kv_len, cu, max_new=max(1, max(kv_len))), tokens=T)
        torch.cuda.synchronize()
        k, v = k.cpu().numpy().astype(np.float64), v.cpu().numpy().astype(np.float64)
        for b, n in enumerate(kv_len):
            for got, want in zip((k, v), self.host.tokens(self.table[b], n, self.slots[b])):
                got = got[cu[b]:cu[b + 1]]
                assert np.all(np.abs(got - want) <= np.abs(want) * 2 ** -11 * (1 + 2 ** -11) + 2 ** -25), b


SHAPES = [(64, 16), (64, 64), (128, 16), (128, 32), (128, 64), (256, 32), (256, 64)]


@pytest.mark.parametrize("dim,page", SHAPES)
def test_append_in_pieces(dim, page):
    """Sequences filled in pieces that end inside, at and past the pages' ends: codes, scales and values are those of one token after the other."""
    steps = [[1, 0, page - 1, page, 2 * page + 5], [page - 1, 3, 1, 1, 1], [1, page - 3, 2 * page, 0, page], [2 * page + 1, 1, 1, page - 1, 0],
             [5, 7, 0, 1, 3 * page]]
    total = [sum(s[b] for s in steps) for b in range(5)]
    w = Both(dim + page, total, 3, dim, page)
    length = [0] * 5
    for new in steps:
        length = [a + n for a, n in zip(length, new)]
        w.append(length, new)
        w.check()
        w.check_tokens(length)


@pytest.mark.parametrize("dim,page", SHAPES)
def test_tail_slots_hold_the_open_pages_tokens(dim, page):
    """Bit for bit, of what is in the slot: the tokens of the page that is not full."""
    steps = [[1, page - 1, 3], [page - 1, 2, page], [5, 0, page - 4], [1, page, 2 * page + 7]]
    w = Both(dim * page, [sum(s[b] for s in steps) for b in range(3)], 2, dim, page)
    length = [0] * 3
    for new in steps:
        length = [a + n for a, n in zip(length, new)]
        w.append(length, new)
        k_tail, v_tail = w.dev.k_tail.cpu().numpy(), w.dev.v_tail.cpu().numpy()
        for b, slot in enumerate(w.slots):
            held = length[b] % page
            assert np.array_equal(k_tail[slot, :, :held], w.host.k_tail[slot, :, :held]), (b, length)
            assert np.array_equal(v_tail[slot, :, :, :held], w.host.v_tail[slot, :, :, :held]), (b, length)


def test_append_values_that_are_not_finite():
    """A NaN is held as 0, an infinity as the largest value, closed or not; other tokens of the page keep their values' scale."""
    w = Both(3, [40], 2, 64, 16)
    k, v = w.random(40)
    k[3, 0, 5], k[20, 1, 6], v[7, 1, 0], v[36, 0, 1], v[37, 0, 2] = np.nan, np.inf, -np.inf, np.nan, np.inf
    w.append([40], [40], k, v)
    w.check()
    w.check_tokens([40])


def test_append_zeros_and_extremes():
    w = Both(4, [32 * 3], 2, 128, 32)
    k, v = w.random(96)
    k[:32], v[32:64], k[64:], v[64:] = 0, 0, k[64:] * np.float16(6e-8), np.sign(v[64:]) * np.float16(65504)
    w.append([96], [96], k, v)
    w.check()
    w.check_tokens([96])


def test_step_between_lengths_of_zero():
    """No sequence, no new token, no token at all."""
    w = Both(5, [70, 10], 1, 64, 64)
    w.append([0, 0], [0, 0])
    w.append([0, 10], [0, 10])
    w.append([70, 10], [70, 0])
    w.check_tokens([70, 10])
    out, _ = qqq.qqq_attention_kv8(w.dev, w.batch([70, 10], [0, 0, 0]), torch.empty(0, 4, 64, dtype=torch.float16, device="cuda"))
    assert out.shape == (0, 4, 64)


def _check_attention(w, kv_len, new, q_heads, scale=None, causal=True, window=0, spread=1.0):
    cu = np.concatenate([[0], np.cumsum(new)])
    T, D = int(cu[-1]), w.dim
    q = (w.rng.standard_normal((T, q_heads, D)) * spread).astype(np.float16)
    wide = torch.full((T, q_heads + 2, D + 8), 5.0, dtype=torch.float16, device="cuda")
    wide[:, 1:-1, :D] = _dev(q)
    out = torch.full((T, q_heads, D), float("nan"), dtype=torch.float16, device="cuda")
    lse = torch.full((T, q_heads), float("nan"), device="cuda")
    qqq.qqq_attention_kv8(w.dev, w.batch(kv_len, cu), wide[:, 1:-1, :D], scale, causal, window, out, lse)
    torch.cuda.synchronize()
    out, lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy()
    scale = D ** -0.5 if scale is None else scale
    for b, n in enumerate(kv_len):
        k, v = w.host.tokens(w.table[b], n, w.slots[b])
        rows = slice(cu[b], cu[b + 1])
        want, want_lse, mag, big = ref.attention(q[rows], k, v, scale, causal, window)
        ds = (D + 8) * 2.0 ** -23 * big
        bound = (2 ** -11 + 2 * ds[..., None] + 3e-5) * mag + n * 2.0 ** -31 * np.abs(v).max(initial=0) + 2 ** -11 * np.abs(want) + 2 ** -25
        worst = (np.abs(out[rows] - want) / bound).max(initial=0)
        assert worst <= 1, (b, n, worst)
        empty = np.isinf(want_lse)
        assert np.array_equal(np.isneginf(lse[rows]), empty)
        assert not out[rows][empty].any()
        assert np.all(np.abs(lse[rows][~empty] - want_lse[~empty]) <= (ds + 3e-5)[~empty]), b


def _filled(seed, lengths, heads, dim, page):
    w = Both(seed, lengths, heads, dim, page)
    w.append(lengths, lengths)
    return w


# lengths: one token, inside a page, at a page's end, inside and at a tile's end, several tiles; a sequence without tokens
LENGTHS = [1, 15, 16, 0, 63, 64, 65, 200, 257]


@pytest.mark.parametrize("dim,page", SHAPES)
@pytest.mark.parametrize("heads,q_heads", [(1, 1), (2, 16), (3, 15)])
def test_single_tokens(dim, page, heads, q_heads):
    w = _filled(11, LENGTHS, heads, dim, page)
    _check_attention(w, LENGTHS, [min(1, n) for n in LENGTHS], q_heads)


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
@pytest.mark.parametrize("new", [2, 5, 9, 16, 40])
def test_a_few_tokens(dim, page, new):
    """Rows past 16, past 32; more new tokens than a sequence has in some."""
    lengths = [40, 64, 130, 300]
    w = _filled(12, lengths, 2, dim, page)
    _check_attention(w, lengths, [new, min(3, new), new, 1], 6)


@pytest.mark.parametrize("dim,page", [(64, 32), (128, 16), (128, 64), (256, 64)])
@pytest.mark.parametrize("q_heads", [2, 14])
def test_prompts(dim, page, q_heads):
    lengths = [1, 129, 200, 64, 333]
    w = _filled(13, lengths, 2, dim, page)
    _check_attention(w, lengths, [1, 129, 77, 64, 333], q_heads)


@pytest.mark.parametrize("window", [1, 16, 50, 64, 1000])
@pytest.mark.parametrize("new", [1, 7, 150])
def test_windows(window, new):
    lengths = [150, 290, 191]
    w = _filled(14, lengths, 2, 128, 32)
    _check_attention(w, lengths, [new, new, min(new, 3)], 8, window=window)


@pytest.mark.parametrize("lengths,new,q_heads,window", [([1024], 1, 64, 1000), ([512], 1, 64, 480), ([512], 1, 32, 500), ([2048], 1, 64, 2000), ([1024, 1024], 1, 64, 1000),
                                                        ([512], 40, 64, 440), ([3827, 90, 3000], 3, 64, 3799)])
def test_windows_a_little_shorter_than_the_past(lengths, new, q_heads, window):
    """The bound of the lengths is that of the window's last whole tile: no more pieces than the workspace query, which knows no window, counts."""
    w = _filled(32, lengths, 8, 128, 64)
    w.max_len = max(lengths)
    _check_attention(w, lengths, [new] * len(lengths), q_heads, window=window)


@pytest.mark.parametrize("new", [1, 6, 60])
def test_without_a_causal_mask(new):
    lengths = [60, 130, 100]
    w = _filled(15, lengths, 2, 64, 16)
    _check_attention(w, lengths, [new] * 3, 6, causal=False)


@pytest.mark.parametrize("new", [1, 3, 40])
def test_rows_that_see_nothing(new):
    """More queries than the sequence has tokens: those before position 0 see nothing."""
    lengths = [0, 2, 33]
    w = _filled(16, lengths, 2, 128, 16)
    _check_attention(w, lengths, [new, max(new, 3), new], 4)


def test_large_scores_and_scales_of_very_different_pages():
    w = Both(17, [256, 256], 2, 128, 16)
    k, v = w.random(512)
    v = (v.astype(np.float64) * np.exp(3 * w.rng.standard_normal((32, 1, 1, 1))).repeat(16, 0).reshape(512, 1, 1)).clip(-6e4, 6e4).astype(np.float16)
    v[64:80] = 0
    k[96:112] = 0
    w.append([256, 256], [256, 256], k, v)
    w.check()
    _check_attention(w, [256, 256], [1, 1], 4, spread=10)
    _check_attention(w, [256, 256], [60, 60], 4, spread=10)
    _check_attention(w, [256, 256], [60, 60], 4, scale=3.0)


def _small_values_beside(seed, dim, page, length, size, lead, first, last):
    """One sequence with values of one sign, `size` in magnitude, whose tokens first .. last - 1 score `lead` (natural logarithm) above the others' mean
    for every query -> (cache, queries' common part).  (Bounds that announce far more, so that many tiles are one wave's.)"""
    w = Both(seed, [length], 1, dim, page, columns=1 << 15)
    k, v = (w.rng.standard_normal((length, 1, dim)) * 0.1).astype(np.float16), (size * (0.5 + 0.5 * w.rng.random((length, 1, dim)))).astype(np.float16)
    toward = np.where(w.rng.random(dim) < 0.5, -1.0, 1.0)
    k[first:last, 0] += (toward * lead / dim ** 0.5).astype(np.float16)
    return w, k, v, toward


def _check_given_queries(w, length, q):
    """As _check_attention, of the last tokens' given queries of one sequence."""
    n, q_heads, D = q.shape
    out, lse = qqq.qqq_attention_kv8(w.dev, w.batch([length], [0, n]), _dev(q), lse=torch.empty(n, q_heads, device="cuda"))
    torch.cuda.synchronize()
    out, lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy()
    k, v = w.host.tokens(w.table[0], length, w.slots[0])
    want, want_lse, mag, big = ref.attention(q, k, v, D ** -0.5)
    ds = (D + 8) * 2.0 ** -23 * big
    bound = (2 ** -11 + 2 * ds[..., None] + 3e-5) * mag + length * 2.0 ** -31 * np.abs(v).max() + 2 ** -11 * np.abs(want) + 2 ** -25
    assert (np.abs(out - want) / bound).max() <= 1, (np.abs(out - want) / bound).max()
    assert np.all(np.abs(lse - want_lse) <= ds + 3e-5)


@pytest.mark.parametrize("size", [1.0, 1e-3, 1e-4])
@pytest.mark.parametrize("dim,page,new,q_heads", [(64, 64, 1, 2), (128, 16, 3, 2), (128, 64, 40, 1), (64, 16, 150, 1), (256, 32, 40, 1)])
def test_small_values_beside_a_page_of_zeros(dim, page, new, q_heads, size):
    """Zeros that score far higher than the values: what the values add is as exact as without them."""
    length = 4096
    w, k, v, toward = _small_values_beside(33, dim, page, length, size, 10.0, 2048, 2048 + page)
    v[2048:2048 + page] = 0
    w.append([length], [length], k, v)
    w.check()
    _check_given_queries(w, length, (toward + 0.1 * w.rng.standard_normal((new, q_heads, dim))).astype(np.float16))


@pytest.mark.parametrize("size", [1.0, 1e-3, 1e-4, 1e4])
@pytest.mark.parametrize("dim,page,length,new,q_heads", [(64, 16, 4017, 1, 2), (128, 16, 4017, 3, 2), (128, 32, 4001, 1, 16), (128, 64, 4020, 1, 2), (64, 16, 4017, 40, 1), (128, 32, 4001, 40, 2),
                                                         (128, 64, 4020, 40, 1), (256, 16, 4017, 1, 20), (256, 32, 4001, 40, 1)])
def test_small_values_beside_an_open_page(dim, page, length, new, q_heads, size):
    """The tail slot's tokens score far higher than the closed pages before them, in the same tile and others: those add what they should."""
    w, k, v, toward = _small_values_beside(34, dim, page, length, size, 10.0, length // page * page, length)
    w.append([length], [length], k, v)
    _check_given_queries(w, length, (toward + 0.1 * w.rng.standard_normal((new, q_heads, dim))).astype(np.float16))


@pytest.mark.parametrize("new,heads,q_heads", [(1, 1, 8), (3, 2, 8), (20, 1, 8), (150, 1, 1)])
def test_a_long_past(new, heads, q_heads):
    """The keys are split over workgroups and joined."""
    lengths = [5000, 700, 3, 4097]
    w = _filled(18, lengths, heads, 64, 64)
    _check_attention(w, lengths, [new, new, min(new, 3), new], q_heads)
    assert "join" in qqq.last_route()
    _check_attention(w, lengths, [new, new, min(new, 3), new], q_heads, window=2000)


@pytest.mark.parametrize("dim,new,q_heads", [(64, 130, 8), (128, 33, 32), (256, 1030, 1)])
def test_many_rows_of_many_splits(dim, new, q_heads):
    """More than eight splits of 1024 rows and more: a wave joins a row's, eight at a time."""
    w = _filled(24, [2700], 1, dim, 64)
    _check_attention(w, [2700], [new], q_heads)
    splits = int(qqq.last_route().split(" x")[1].split()[0])
    assert splits > 8 and "join" in qqq.last_route()
    _check_attention(w, [2700], [new], q_heads, window=2300)


@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("q_heads", [1, 9])
def test_equal_shares_of_many_sequences(q_heads, window):
    """More sequences than a workgroup has threads, long, short and empty, some without a new token: shares begin and end inside of them."""
    rng = np.random.default_rng(26)
    lengths = [int(n) for n in rng.integers(0, 150, 300)]
    lengths[7], lengths[8], lengths[200], lengths[299] = 2500, 0, 3333, 64
    new = [int(rng.integers(0, 4)) for _ in lengths]
    new[7], new[8], new[199], new[200], new[299] = 3, 2, 0, 1, 1
    w = _filled(27, lengths, 1, 64, 64)
    _check_attention(w, lengths, new, q_heads, window=window)
    if not window:
        assert "rows x512 + join" in qqq.last_route()


@pytest.mark.parametrize("lengths,new", [([5, 0, 70], [1, 1, 1]), ([0, 0, 0], [1, 2, 0]), ([1, 900, 3], [0, 4, 0]), ([640, 640, 640], [1, 1, 1]), ([257, 1, 512], [2, 1, 1])])
def test_equal_shares_of_less_than_was_announced(lengths, new):
    """Bounds that promise far more tokens than there are: most shares are empty."""
    w = Both(28, lengths, 8, 128, 64, columns=1100)
    w.append(lengths, lengths)
    _check_attention(w, lengths, new, 32)
    assert "rows x64 + join" in qqq.last_route()


@pytest.mark.parametrize("dim,page", SHAPES + [(256, 16), (64, 32)])
@pytest.mark.parametrize("new", [1, 4])
def test_equal_shares_of_every_shape(dim, page, new):
    """Shares that end inside of sequences, with tail slots beside pages shorter than a tile; 7 and 28 rows of a head."""
    lengths = [300, 0, 129 + page, 64, 700]
    w = Both(29, lengths, 2, dim, page, columns=900 * 64 // page)
    w.append(lengths, lengths)
    _check_attention(w, lengths, [min(new, n) for n in lengths], 14)
    assert "rows x256 + join" in qqq.last_route()


@pytest.mark.parametrize("dim,page", SHAPES + [(256, 16), (64, 32)])
@pytest.mark.parametrize("new", [1, 4, 40])
@pytest.mark.parametrize("announced", [1100, 70000, 1 << 21])
def test_one_sequence_of_every_shape(dim, page, new, announced):
    """7, 28 and 280 rows of a head, by what the bounds announce whole, in pieces, and in many; the last tokens in the tail slot."""
    w = Both(31, [1000], 2, dim, page, columns=announced // page)
    w.append([1000], [1000])
    _check_attention(w, [1000], [new], 14)
    _check_attention(w, [1000], [new], 14, window=100)


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (128, 64)])
@pytest.mark.parametrize("new", [1, 17])
def test_one_long_sequence_of_many_heads(dim, page, new):
    w = _filled(30, [4200], 32, dim, page)
    _check_attention(w, [4200], [new], 32)
    assert "join" in qqq.last_route()


def test_more_values_than_the_last_level_cache():
    """A call that goes past the caches: the same bits as in pieces that do not."""
    H, D, P, n = 40, 128, 16, 9000
    pages = n // P
    table = torch.randperm(pages, device="cuda").int().view(1, -1)
    k, v = (torch.randn(n, H, D, device="cuda").half() for _ in range(2))
    whole, pieces = (qqq.new_kv8_cache(pages, H, D, P, 1) for _ in range(2))
    step = lambda length, new: qqq.KV8Batch(table, torch.tensor([length], dtype=torch.int32, device="cuda"),  # noqa: E731
                                            torch.tensor([0, new], dtype=torch.int32, device="cuda"), None, new, n)
    qqq.qqq_kv8_append(whole, step(n, n), k, v)
    for at in range(0, n, 3000):
        qqq.qqq_kv8_append(pieces, step(at + 3000, 3000), k[at:at + 3000], v[at:at + 3000])
    torch.cuda.synchronize()
    for name in ("k_codes", "k_scale", "v_codes", "v_scale", "k_tail", "v_tail"):
        assert torch.equal(getattr(whole, name), getattr(pieces, name)), name
    got = qqq.qqq_kv8_read(whole, step(n, n), tokens=n)
    for at in (3000, 6000):  # (3000 tokens end inside a page, whose place in the tail slot is another's by now)
        for a, b in zip(got, qqq.qqq_kv8_read(pieces, step(at + 3000, 3000), tokens=3000)):
            assert torch.equal(a[at:at + 3000], b), at


@pytest.mark.parametrize("new,length", [(1, 40), (1, 700), (1, 5000), (40, 100), (40, 2000), (300, 3500)])
def test_a_query_that_is_not_a_number(new, length):
    """It gives NaN in its own row, in what the sum's logarithm is as well, whole or joined from splits."""
    w = _filled(25, [length], 1, 64, 64)
    q = torch.randn(new, 4, 64, device="cuda").half()
    batch = w.batch([length], [0, new])
    want, want_lse = torch.empty_like(q), torch.empty(new, 4, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(new, 4, device="cuda")
    qqq.qqq_attention_kv8(w.dev, batch, q, out=want, lse=want_lse)
    q[new // 2, 2, 7] = float("nan")
    qqq.qqq_attention_kv8(w.dev, batch, q, out=out, lse=lse)
    torch.cuda.synchronize()
    here = torch.zeros(new, 4, dtype=torch.bool, device="cuda")
    here[new // 2, 2] = True
    assert out[here].isnan().all() and lse[here].isnan().all()
    assert torch.isfinite(out[~here]).all()
    # (the many-rows kernel may take another reference for the rows beside it: as far from the formula's as before)
    assert (out[~here].float() - want[~here].float()).abs().max() <= 2 ** -9 * want.float().abs().max()
    assert (lse[~here] - want_lse[~here]).abs().max() <= 1e-4


def test_same_result_twice_and_on_another_stream():
    w = _filled(19, [3000, 100], 2, 128, 64)
    q = torch.randn(2, 16, 128, device="cuda").half()
    batch = w.batch([3000, 100], [0, 1, 2])
    first, _ = qqq.qqq_attention_kv8(w.dev, batch, q)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        second, _ = qqq.qqq_attention_kv8(w.dev, batch, q)
    stream.synchronize()
    assert torch.equal(first, second)


def test_graph_of_a_step_replayed_with_other_lengths():
    """A captured step reads lengths on the device: each replay equals calls of its own on another cache."""
    lengths = [130, 64, 200]
    a, b = _filled(20, lengths, 2, 64, 64), _filled(20, lengths, 2, 64, 64)
    start = [126, 62, 190]
    kv_len = _dev(np.array(start, np.int32))
    cu = _dev(np.arange(4, dtype=np.int32))
    batch = qqq.KV8Batch(_dev(a.table), kv_len, cu, _dev(a.slots), 1, a.max_len)
    for w in (a, b):
        k, v = w.random(sum(start))
        w.append(start, start, k, v)
    kv = torch.zeros(3, 2, 2, 64, dtype=torch.float16, device="cuda")
    q, out = torch.zeros(3, 8, 64, dtype=torch.float16, device="cuda"), torch.zeros(3, 8, 64, dtype=torch.float16, device="cuda")
    work = torch.empty(max(1, qqq.qqq_attention_kv8_workspace_bytes(a.dev, batch, 8, 3)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv_len += 1
        qqq.qqq_kv8_append(a.dev, batch, kv[:, 0], kv[:, 1])
        qqq.qqq_attention_kv8(a.dev, batch, q, out=out, workspace=work)
    kv_len.copy_(_dev(np.array(start, np.int32)))
    for step in range(4):
        kv.copy_(torch.randn(3, 2, 2, 64, device="cuda"))
        q.copy_(torch.randn(3, 8, 64, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        now = [n + step + 1 for n in start]
        other = qqq.KV8Batch(_dev(b.table), _dev(np.array(now, np.int32)), cu, _dev(b.slots), 1, b.max_len)
        qqq.qqq_kv8_append(b.dev, other, kv[:, 0], kv[:, 1])
        want, _ = qqq.qqq_attention_kv8(b.dev, other, q)
        torch.cuda.synchronize()
        assert torch.equal(out, want), step
        assert torch.equal(a.dev.k_codes, b.dev.k_codes) and torch.equal(a.dev.v_codes, b.dev.v_codes)


def test_device_tables_out_of_bounds_stay_inside():
    """Lengths, rows, pages and slots that the host's bounds rule out are cut, skipped or replaced on the device: nothing outside is written."""
    w = _filled(21, [64, 32], 1, 64, 16)
    before = [t.clone() for t in w.dev]
    table = _dev(np.array([[1 << 30, -7, 3, 99], [5, 6, 1000, -1]], np.int32))
    kv = torch.randn(20, 2, 1, 64, device="cuda").half()
    q = torch.randn(20, 4, 64, device="cuda").half()
    for kv_len, cu, slots in (([1 << 30, -5], [0, 9, 20], [0, 1]), ([64, 32], [-3, 17, 400], [77, -1]), ([64, 32], [0, -4, 1 << 30], [0, 1])):
        batch = qqq.KV8Batch(table, _dev(np.array(kv_len, np.int32)), _dev(np.array(cu, np.int32)), _dev(np.array(slots, np.int32)), 16, 4 * 16 + 15)
        out, _ = qqq.qqq_attention_kv8(w.dev, batch, q)
        qqq.qqq_kv8_read(w.dev, batch, tokens=20)
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, w.dev))
    qqq.qqq_kv8_append(w.dev, qqq.KV8Batch(table, _dev(np.array([64, 32], np.int32)), _dev(np.array([0, 9, 20], np.int32)),
                                           _dev(np.array([77, -1], np.int32)), 16, 79), kv[:, 0], kv[:, 1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, w.dev))


def test_caches_whose_offsets_pass_32_bits():
    """The same pages at the end of a cache of over 4 GiB of codes as at the start of a small one: append, read and attention give the same bits."""
    H, D, P, B = 8, 128, 64, 2
    pages = (1 << 32) // (H * D * P) + 40
    rng = np.random.default_rng(22)
    lengths = [300, 129]
    order = rng.permutation(12)
    i32 = lambda a: _dev(np.asarray(a, np.int32))  # noqa: E731
    tables = [np.concatenate([order[:4], order[4:8]]).reshape(2, 4), pages - 1 - np.concatenate([order[:4], order[4:8]]).reshape(2, 4)]
    k, v = (torch.randn(sum(lengths), H, D, device="cuda").half() for _ in range(2))
    q1, q2 = torch.randn(2, 16, D, device="cuda").half(), torch.randn(sum(lengths), 16, D, device="cuda").half()
    got = []
    for table, n in zip(tables, (12, pages)):
        cache = qqq.KV8Cache(torch.empty(n, H, P, D, dtype=torch.uint8, device="cuda"), torch.empty(n, H, device="cuda"), torch.empty(n, H, D, P, dtype=torch.uint8, device="cuda"),
                             torch.empty(n, H, device="cuda"), *(torch.zeros(B, H, *s, dtype=torch.float16, device="cuda") for s in ((P, D), (D, P))))
        assert n == 12 or cache.k_codes.numel() > 1 << 32
        whole = qqq.KV8Batch(i32(table), i32(lengths), i32([0, 300, 429]), None, 300, 300)
        qqq.qqq_kv8_append(cache, whole, k, v)
        one, _ = qqq.qqq_attention_kv8(cache, whole._replace(cu=i32([0, 1, 2]), max_new=1), q1)
        many, _ = qqq.qqq_attention_kv8(cache, whole, q2)
        got.append((*qqq.qqq_kv8_read(cache, whole, tokens=429), one, many))
        torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_marshalled_in_python(monkeypatch):
    """Without the extension the calls are the same, refusals included."""
    w = _filled(23, [100, 40], 2, 64, 32)
    batch = w.batch([100, 40], [0, 3, 5])
    q, kv = torch.randn(5, 4, 64, device="cuda").half(), torch.randn(5, 2, 64, device="cuda").half()
    lse = [torch.empty(5, 4, device="cuda") for _ in range(2)]
    x, r, gain = torch.randn(5, 256, device="cuda").half(), torch.randn(5, 256, device="cuda"), torch.ones(256, device="cuda").half()

    def all_calls(i):
        qqq.qqq_kv8_append(w.dev, batch, kv, kv)   # (no page is filled by it: it can be done again)
        outs = [*qqq.qqq_attention_kv8(w.dev, batch, q, lse=lse[i]), *qqq.qqq_kv8_read(w.dev, batch, *(torch.empty(5, 2, 64, device="cuda").half() for _ in range(2)))]
        outs += [*qqq.qqq_add_rmsnorm(x, gain, r), *qqq.qqq_add_rmsnorm_quant(x, gain, r), *qqq.qqq_add_rmsnorm_quant(x, gain)[1:], *qqq.qqq_gated_act_quant(x, r.half(), "gelu_tanh")]
        torch.cuda.synchronize()
        return [t.clone() for t in outs] + [t.clone() for t in w.dev]

    def refusals():
        with pytest.raises(ValueError):
            qqq.qqq_add_rmsnorm(x, gain[:100])
        with pytest.raises(ValueError):
            qqq.qqq_gated_act_quant(x, r)
        with pytest.raises(ValueError):
            qqq.qqq_attention_kv8(w.dev, batch, q[..., :32])
        with pytest.raises(ValueError):
            qqq.qqq_kv8_append(w.dev, batch, kv, kv[:4])
        with pytest.raises(ValueError):
            qqq.qqq_kv8_append(w.dev._replace(k_scale=w.dev.k_scale[:1]), batch, kv, kv)
        for call in (lambda: qqq.qqq_add_rmsnorm_quant(x, gain, r, eps=-1.0), lambda: qqq.qqq_attention_kv8(w.dev, batch, q[:, :3].contiguous()),
                     lambda: qqq.qqq_attention_kv8(w.dev, batch._replace(max_len=1000), q), lambda: qqq.qqq_attention_kv8(w.dev, batch, q, window=4, causal=False),
                     lambda: qqq.qqq_add_rmsnorm(torch.empty(5 * 256 + 1, device="cuda").half()[1:].view(5, 256), gain)):
            with pytest.raises(qqq.QQQError) as e:
                call()
            assert e.value.code == 2
    first = all_calls(0)
    refusals()
    for name in ("rmsnorm", "gated", "append", "read", "attention"):
        monkeypatch.setattr(qqq, "_native_" + name, qqq._no_native)
    second = all_calls(1)
    refusals()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
