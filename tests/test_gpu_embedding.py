"""Embedding rows and their gradient against plain sums in 64 bits."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_1910_04940_amd as bl  # noqa: E402

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # largest relative error of a rounding


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _tokens(kind, n, vocab, seed, dtype=torch.int64):
    rng = np.random.default_rng(seed)
    t = {"spread": lambda: rng.integers(0, vocab, n), "uneven": lambda: np.minimum(vocab - 1, (vocab ** rng.random(n)).astype(np.int64) - 1),
         "one": lambda: np.full(n, vocab // 2), "ends": lambda: rng.choice([0, vocab - 1], n),
         "padded": lambda: np.where(np.arange(n) < n - n // 3, rng.integers(0, vocab, n), rng.choice([-1, vocab, vocab + 7, -2 ** 31], n)),
         "padding": lambda: np.full(n, -1), "rising": lambda: np.sort(rng.integers(0, vocab, n))}[kind]()
    return torch.from_numpy(t.astype(np.int64)).to(dtype).cuda()


def _want_rows(table, tokens, scale, dtype):
    ok = (tokens >= 0) & (tokens < table.shape[0])
    at = torch.where(ok, tokens, 0).long()
    return torch.where(ok[:, None], table[at].float() * scale, 0.0).to(dtype)   # one multiplication and one rounding, as there


@pytest.mark.parametrize("table_type", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("out_type", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,vocab,dim,kind", [(1, 1, 1, "one"), (1, 50, 4096, "one"), (7, 3, 8, "padded"), (1001, 777, 33, "padded"), (300, 1000, 512, "spread"),
                                              (64, 100, 1000, "padding"), (5000, 200, 24, "uneven")])
def test_rows(n, vocab, dim, kind, table_type, out_type):
    g = torch.Generator("cuda").manual_seed(3)
    table = torch.randn(vocab, dim, generator=g, device="cuda").to(table_type)
    for dtype in (torch.int32, torch.int64):
        tokens = _tokens(kind, n, vocab, 5, dtype)
        out = torch.full((n, dim), 7.0, device="cuda").to(out_type)
        bl.blink_embedding(table, tokens, out, 0.7, _stream())
        assert torch.equal(out, _want_rows(table, tokens, 0.7, out_type))


@pytest.mark.parametrize("shift,pad", [(0, 8), (8, 8), (1, 8), (0, 3), (0, 0)])
def test_rows_at_any_stride_and_alignment(shift, pad):
    """Views into wider tables; what lies beside the rows of the result stays."""
    vocab, dim, n = 90, 64, 133
    wide = torch.randn(vocab, dim + shift + pad, device="cuda").bfloat16()
    tokens = _tokens("padded", n, vocab, 6)
    whole = torch.full((n, dim + shift + pad), 5.0, dtype=torch.bfloat16, device="cuda")
    bl.blink_embedding(wide[:, shift:shift + dim], tokens, whole[:, shift:shift + dim], 2.0, _stream())
    assert torch.equal(whole[:, shift:shift + dim], _want_rows(wide[:, shift:shift + dim], tokens, 2.0, torch.bfloat16))
    beside = torch.cat((whole[:, :shift], whole[:, shift + dim:]), 1)
    assert (beside == 5.0).all()


def test_a_table_past_32_bits():
    """Rows whose offset passes 2^32 bytes and 2^31 elements."""
    vocab, dim = 9_000, 262_144 // 1
    table = torch.empty(vocab, dim, dtype=torch.bfloat16, device="cuda")
    table[8_990:] = torch.randn(10, dim, device="cuda").bfloat16()
    tokens = torch.tensor([8_999, 8_990, 8_195, 9_000], device="cuda")
    table[8_195] = 3.0
    out = torch.empty(4, dim, dtype=torch.bfloat16, device="cuda")
    bl.blink_embedding(table, tokens, out, 1.0, _stream())
    assert torch.equal(out[:2], table[[8_999, 8_990]]) and (out[2] == 3.0).all() and (out[3] == 0).all()


def test_infinities_and_nan_of_rows_that_nobody_names():
    table = torch.randn(10, 16, device="cuda")
    table[0] = float("nan")
    table[9] = float("inf")
    tokens = torch.tensor([1, -1, 10, 8], device="cuda")
    out = torch.empty(4, 16, device="cuda")
    bl.blink_embedding(table, tokens, out, float("inf"), _stream())
    assert (out[1:3] == 0).all() and not torch.isnan(out).any()


def _gradient(tokens, grad, table, scale, accumulate):
    n = tokens.numel()
    work = torch.full((max(1, bl.blink_embedding_gradient_workspace(n, *table.shape)),), 255, dtype=torch.uint8, device="cuda")
    bl.blink_embedding_gradient(tokens, grad, table, work, scale, accumulate, _stream())


def _check(tokens, grad, before, got, scale, accumulate):
    """Any order of adding c numbers in 32 bits is off by at most c units of the sum of their sizes; then one rounding."""
    vocab, dim = got.shape
    tokens, grad = tokens.cpu().long(), grad.cpu().double()
    ok = (tokens >= 0) & (tokens < vocab)
    want, size = (torch.zeros(vocab, dim, dtype=torch.float64) for _ in range(2))
    want.index_add_(0, tokens[ok], grad[ok] * scale)
    size.index_add_(0, tokens[ok], grad[ok].abs() * abs(scale))
    many = torch.bincount(tokens[ok], minlength=vocab)[:, None]
    if accumulate:
        want += before.cpu().double()
        size += before.cpu().double().abs()
    off = (got.cpu().double() - want).abs()
    tiny = 2.0 ** -24 if got.dtype == torch.float16 else 2.0 ** -133
    allowed = (many + 3) * 2.0 ** -24 * size + UNIT[got.dtype] * want.abs() * 1.01 + tiny
    assert (off <= allowed).all(), (off - allowed).max()
    if accumulate:
        same = (many[:, 0] == 0)
        assert torch.equal(got.cpu()[same], before.cpu()[same])
    else:
        assert (got.cpu()[many[:, 0] == 0] == 0).all()


SIZES = [(1, 1, 1, "one"), (1, 1000, 64, "one"), (2, 3, 5, "ends"), (63, 40, 100, "spread"), (64, 64, 256, "rising"), (65, 500, 257, "uneven"),
         (1000, 7, 64, "uneven"), (1025, 3000, 300, "padded"), (8192, 300, 40, "uneven"), (8193, 1000, 64, "uneven"), (20_011, 70_001, 24, "uneven"),
         (5000, 50, 1000, "one"), (30_000, 131_072, 8, "padded"), (9000, 513, 16, "ends"), (700, 90, 33, "padding"), (40_000, 1, 8, "one")]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("grad_type,table_type", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
                                                  (torch.float16, torch.float16), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("n,vocab,dim,kind", SIZES)
def test_gradient(n, vocab, dim, kind, grad_type, table_type, accumulate):
    g = torch.Generator("cuda").manual_seed(n + dim)
    tokens = _tokens(kind, n, vocab, 9, torch.int32 if dim % 2 else torch.int64)
    grad = torch.randn(n, dim, generator=g, device="cuda").to(grad_type)
    before = torch.randn(vocab, dim, generator=g, device="cuda").to(table_type) if accumulate else torch.full((vocab, dim), float("nan"), device="cuda").to(table_type)
    got = before.clone()
    _gradient(tokens, grad, got, 0.5, accumulate)
    _check(tokens, grad, before, got, 0.5, accumulate)
    again = before.clone()
    _gradient(tokens, grad, again, 0.5, accumulate)
    assert torch.equal(got.view(torch.uint8), again.view(torch.uint8))    # the same every time


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,vocab,dim,kind", [(262_144, 3000, 8, "uneven"), (300_001, 600_000, 4, "uneven"), (550_000, 40, 8, "padded"), (9_000, 1 << 20, 4, "spread"),
                                              (262_145, 200, 16, "one")])
def test_gradient_of_long_lists(n, vocab, dim, kind, accumulate):
    """Chunks of several tiles, three sorting passes, one token for all."""
    g = torch.Generator("cuda").manual_seed(n)
    tokens = _tokens(kind, n, vocab, 9)
    grad = torch.randn(n, dim, generator=g, device="cuda")
    before = torch.randn(vocab, dim, generator=g, device="cuda") if accumulate else torch.full((vocab, dim), float("nan"), device="cuda")
    got = before.clone()
    _gradient(tokens, grad, got, 0.5, accumulate)
    _check(tokens, grad, before, got, 0.5, accumulate)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("vocab,dim", [(64, 64), (300, 5), (300_000, 8)])
def test_gradient_of_one_token(vocab, dim, accumulate):
    """Wherever the token's row lies among the places that a wave takes (8 of them for the short tables, 32 for the long one), its
    position and the row's end beside one another or not; and one token that is padding."""
    grad = torch.arange(1.0, dim + 1, device="cuda").reshape(1, dim)
    before = torch.arange(float(vocab), device="cuda")[:, None] + torch.zeros(1, dim, device="cuda") if accumulate else torch.full((vocab, dim), float("nan"), device="cuda")
    wrong = []
    for token in [*range(64), vocab - 2, vocab - 1, vocab, -1]:
        got = before.clone()
        _gradient(torch.tensor([token], device="cuda"), grad, got, 0.5, accumulate)
        want = before.clone() if accumulate else torch.zeros(vocab, dim, device="cuda")
        if 0 <= token < vocab:
            want[token] = want[token] + 0.5 * grad[0]     # halves of small whole numbers: exact
        if not torch.equal(got, want):
            wrong.append(token)
    assert wrong == []


@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_without_tokens(accumulate):
    table = torch.randn(100, 24, device="cuda")
    before = table.clone()
    _gradient(torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, 24, device="cuda"), table, 1.0, accumulate)
    assert torch.equal(table, before if accumulate else torch.zeros_like(before))


def test_gradient_of_one_row_for_all_tokens_and_of_views():
    n, vocab, dim = 3000, 41, 64
    tokens = _tokens("uneven", n, vocab, 11)
    row = torch.randn(1, dim, device="cuda")
    got = torch.empty(vocab, dim, device="cuda")
    _gradient(tokens, row.expand(n, dim), got, 1.0, False)
    _check(tokens, row.expand(n, dim).contiguous(), None, got, 1.0, False)
    wide, whole = torch.randn(n, dim + 9, device="cuda"), torch.full((vocab, dim + 5), 3.0, device="cuda")
    _gradient(tokens, wide[:, 9:], whole[:, :dim], 1.0, False)
    _check(tokens, wide[:, 9:].contiguous(), None, whole[:, :dim].contiguous(), 1.0, False)
    assert (whole[:, dim:] == 3.0).all()


def test_more_rows_than_a_launch_has_threads_in_one_direction():
    """More than 2^33 elements that are loaded one by one: their places pass 32 bits, their workgroups 2^24."""
    n, vocab, dim = 8_600_000, 300, 1001
    table = torch.randn(vocab, dim, device="cuda").bfloat16()
    tokens = torch.from_numpy(np.random.default_rng(7).integers(-1, vocab, n)).cuda()
    out = torch.full((n, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    bl.blink_embedding(table, tokens, out, 1.0, _stream())
    for lo in range(0, n, 500_000):
        assert torch.equal(out[lo:lo + 500_000], _want_rows(table, tokens[lo:lo + 500_000], 1.0, torch.bfloat16))


def test_a_longer_table_than_a_launch_has_threads_in_one_direction():
    """The largest vocabulary: more than 2^24 workgroups, and keys of 31 bits."""
    n, vocab = 3000, (1 << 31) - 2
    rng = np.random.default_rng(8)
    tokens = np.concatenate((rng.integers(0, vocab, n - 1000), rng.integers(vocab - 70, vocab, 900), rng.integers(0, 70, 90), np.full(10, vocab)))
    tokens = torch.from_numpy(rng.permutation(tokens)).cuda()
    grad = torch.randint(-3, 4, (n, 1), device="cuda").bfloat16()
    table = torch.full((vocab, 1), 2.0, dtype=torch.bfloat16, device="cuda")
    _gradient(tokens, grad, table, 0.5, False)
    named = torch.unique(tokens[tokens < vocab])
    want = torch.zeros(len(named), device="cuda").index_add_(0, torch.searchsorted(named, tokens[tokens < vocab]), 0.5 * grad[tokens < vocab, 0].float())
    assert torch.equal(table[named, 0].float(), want)     # small halves: exact
    table[named] = 0.0
    for lo in range(0, vocab, 1 << 28):
        assert (table[lo:lo + (1 << 28)] == 0.0).all()


@pytest.mark.parametrize("accumulate", [False, True])
def test_a_gradient_past_32_bits(accumulate):
    """A table of more than 2^32 elements: the rows that tokens name, and others beside them."""
    vocab, dim, n = 1_100_000, 4096, 3000
    table = torch.full((vocab, dim), 2.0, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(3)
    tokens = torch.from_numpy(np.concatenate([rng.integers(vocab - 500, vocab, n - 1000), rng.integers(0, vocab, 1000)])).cuda()
    grad = torch.randint(-3, 4, (n, dim), device="cuda").bfloat16()
    _gradient(tokens, grad, table, 0.5, accumulate)
    named = torch.unique(tokens)
    want = torch.zeros(len(named), dim, device="cuda").index_add_(0, torch.searchsorted(named, tokens), 0.5 * grad.float()) + (2.0 if accumulate else 0.0)
    assert torch.equal(table[named].float(), want)      # small whole numbers and halves: exact
    others = torch.ones(vocab, dtype=torch.bool, device="cuda")
    others[named] = False
    for lo in range(0, vocab, 100_000):
        part = others[lo:lo + 100_000]
        assert (table[lo:lo + 100_000][part] == (2.0 if accumulate else 0.0)).all()


def test_padding_keeps_nan_out():
    tokens = torch.tensor([0, -1, 2, 5, 0], device="cuda")
    grad = torch.ones(5, 8, device="cuda")
    grad[1] = float("nan")
    grad[3] = float("inf")
    got = torch.empty(4, 8, device="cuda")
    _gradient(tokens, grad, got, 1.0, False)
    assert got[:, 0].tolist() == [2.0, 0.0, 1.0, 0.0]


def test_gradient_against_differences():
    """The gradient of f(table) = sum of c * rows(table), by changing entries of the table: f is linear, so exactly."""
    vocab, dim, n, scale = 9, 8, 40, 0.5
    tokens = _tokens("padded", n, vocab, 13)
    c = torch.randint(-4, 5, (n, dim), device="cuda").float()
    got = torch.empty(vocab, dim, device="cuda")
    _gradient(tokens, c, got, scale, False)
    table = torch.randint(-8, 9, (vocab, dim), device="cuda").float()
    out = torch.empty(n, dim, device="cuda")

    def f(t):
        bl.blink_embedding(t, tokens, out, scale, _stream())
        return float((c * out).sum())
    for v in range(vocab):
        for d in (0, 3, 7):
            up, down = table.clone(), table.clone()
            up[v, d] += 1
            down[v, d] -= 1
            assert (f(up) - f(down)) / 2 == got[v, d]


def test_on_another_stream_and_in_a_graph():
    n, vocab, dim = 9000, 500, 64
    tokens = _tokens("uneven", n, vocab, 17)
    grad = torch.randn(n, dim, device="cuda")
    want = torch.empty(vocab, dim, device="cuda")
    _gradient(tokens, grad, want, 1.0, False)
    work = torch.empty(bl.blink_embedding_gradient_workspace(n, vocab, dim), dtype=torch.uint8, device="cuda")
    got, rows = torch.empty_like(want), torch.empty(n, dim, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bl.blink_embedding_gradient(tokens, grad, got, work, 1.0, False, _stream())
        bl.blink_embedding(got, tokens, rows, 1.0, _stream())
    for _ in range(3):
        got.fill_(9.0)
        rows.fill_(9.0)
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(rows, want[tokens])


def test_c_status_comes_back_as_an_error():
    with pytest.raises(bl.BlinkError) as e:
        bl.blink_embedding_gradient(torch.zeros(5, dtype=torch.int64, device="cuda"), torch.zeros(5, 8, device="cuda"), torch.zeros(9, 8, device="cuda"),
                                    torch.zeros(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == bl.BLINK_EINVAL
    assert C.sizeof(C.c_size_t) == 8
