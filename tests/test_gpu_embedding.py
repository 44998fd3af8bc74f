"""The embedding's lookup and its gradient against plain sums in 64 bits on the CPU."""
import numpy as np
import pytest
import torch

from paper_2305_12201_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _matrix(rows, cols, dtype, seed, extra=0, shift=0, sigma=1.0):
    """A matrix on the GPU whose rows lie `extra` elements apart and which starts `shift` elements into its buffer; the
    elements between the rows are NaN."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((shift + rows * (cols + extra),), float("nan"), dtype=dtype)
    m = buf[shift:].view(rows, cols + extra)[:, :cols]
    m.copy_((torch.randn(rows, cols, generator=g) * sigma).to(dtype))
    buf = buf.cuda()
    return buf, buf[shift:].view(rows, cols + extra)[:, :cols]


def _tokens(n, vocab, dtype, seed, kind="text"):
    g = torch.Generator().manual_seed(seed)
    if kind == "text":      # a few frequent ones, many rare ones
        u = torch.rand(n, generator=g, dtype=torch.float64)
        t = (vocab ** u - 1).floor().clamp(0, vocab - 1)
    elif kind == "uniform":
        t = torch.randint(0, vocab, (n,), generator=g)
    elif kind == "same":
        t = torch.full((n,), vocab - 1)
    elif kind == "none":
        t = torch.full((n,), -1)
    else:                   # "padded": in places no token, in places one that does not exist
        t = torch.randint(0, vocab, (n,), generator=g)
        t[::3] = -1
        t[1::7] = vocab
        t[2::11] = torch.iinfo(dtype).max - 2
        if dtype == torch.int64:
            t[5::13] = (1 << 32) + 1     # a token whose low 32 bits would be one
            t[6::13] = -(1 << 40)
    return t.to(dtype)


# ---- lookup ---------------------------------------------------------------------------------------------------------

def _expected_lookup(table, tokens, scale, dtype):
    """The product rounded to binary32, then to the output's type: the same two roundings as specified, bit for bit."""
    t, V = tokens.long(), table.shape[0]
    ok = (t >= 0) & (t < V)
    rows = table[t.clamp(0, V - 1)].float() * np.float32(scale).item()
    return torch.where(ok[:, None], rows, torch.zeros(())).to(dtype)


@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 50, 4096), (3, 7, 5), (64, 1000, 64), (700, 3000, 650), (513, 100, 1031),
                                         (5000, 300, 770), (20_001, 9, 12), (2, 3, 70_001)])
@pytest.mark.parametrize("dtype", TYPES)
def test_lookup(n, vocab, dim, dtype):
    _, table = _matrix(vocab, dim, dtype, 1)
    for itype, kind, scale in ((torch.int64, "padded", 1.0), (torch.int32, "text", 0.3)):
        tokens = _tokens(n, vocab, itype, 2, kind)
        out = torch.full((n, dim), float("nan"), dtype=dtype, device="cuda")
        B.gravac_embedding_lookup(table, tokens.cuda(), out, scale=scale)
        want = _expected_lookup(table.cpu(), tokens, scale, dtype)
        assert torch.equal(out.cpu().view(torch.int16 if dtype != torch.float32 else torch.int32),
                           want.view(torch.int16 if dtype != torch.float32 else torch.int32)), (kind, scale)


@pytest.mark.parametrize("a", TYPES)
@pytest.mark.parametrize("b", TYPES)
def test_lookup_types_strides_and_odd_starts(a, b):
    n, vocab, dim = 77, 40, 203
    _, table = _matrix(vocab, dim, a, 3, extra=5, shift=1)
    buf, out = _matrix(n, dim, b, 4, extra=3, shift=1)
    before = buf.cpu().clone()
    tokens = _tokens(n, vocab, torch.int64, 5, "padded")
    B.gravac_embedding_lookup(table, tokens.cuda(), out, scale=2.5)
    want = _expected_lookup(table.cpu(), tokens, 2.5, b)
    got = buf.cpu()
    m = got[1:].view(n, dim + 3)
    assert torch.equal(m[:, :dim], want)
    # what lies between the rows is left as it was
    assert torch.isnan(m[:, dim:]).all() and torch.isnan(got[:1]).all() and torch.isnan(before[1:].view(n, dim + 3)[:, dim:]).all()


def test_lookup_special_values():
    table = torch.tensor([[float("inf"), -float("inf"), float("nan"), 3.0e38, -0.0, 1e-45]], dtype=torch.float32, device="cuda")
    tokens = torch.tensor([0, -1, 1, 0], device="cuda")
    out = torch.full((4, 6), 7.0, dtype=torch.float32, device="cuda")
    B.gravac_embedding_lookup(table, tokens, out, scale=2.0)
    x = out.cpu()
    for r in (0, 3):
        assert x[r, 0] == float("inf") and x[r, 1] == -float("inf") and torch.isnan(x[r, 2]) and x[r, 3] == float("inf")
        assert x[r, 4] == 0 and torch.signbit(x[r, 4]) and x[r, 5] == np.float32(2.8e-45)
    assert torch.equal(x[1:3].view(torch.int32), torch.zeros(2, 6, dtype=torch.int32))     # +0, whatever row 0 holds
    out = torch.full((4, 6), 7.0, dtype=torch.float32, device="cuda")
    B.gravac_embedding_lookup(table, tokens, out, scale=float("inf"))
    assert torch.equal(out.cpu()[1:3].view(torch.int32), torch.zeros(2, 6, dtype=torch.int32))


def test_lookup_behind_32_bits():
    vocab, dim = 600_001, 4096                       # 2.46e9 elements
    table = torch.zeros(vocab, dim, dtype=torch.bfloat16, device="cuda")
    rows = [0, 524_287, 524_288, 600_000]
    for i, r in enumerate(rows):
        table[r] = i + 1
    out = torch.empty(4, dim, dtype=torch.bfloat16, device="cuda")
    B.gravac_embedding_lookup(table, torch.tensor(rows, dtype=torch.int32, device="cuda"), out)
    assert torch.equal(out.cpu(), torch.arange(1, 5).to(torch.bfloat16)[:, None].expand(4, dim))


# ---- gradient -------------------------------------------------------------------------------------------------------

def _gradient(grad_out, tokens, table, padding=-1, scale=1.0, accumulate=False, ws=None):
    if ws is None:
        size = B.gravac_embedding_gradient_workspace_bytes(tokens.numel(), *table.shape)
        ws = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
    B.gravac_embedding_gradient(grad_out, tokens, table, scale=scale, padding_token=padding, accumulate=accumulate, workspace=ws)


def _expected_gradient(grad_out, tokens, vocab, padding, scale):
    """Per entry: the sum in 64 bits, the sum of magnitudes and the number of terms of its row."""
    t = tokens.long()
    ok = (t >= 0) & (t < vocab) & (t != padding)
    x = grad_out.double()[ok]
    s = np.float32(scale).item()
    total = torch.zeros(vocab, grad_out.shape[1], dtype=torch.float64).index_add_(0, t[ok], x) * s
    size = torch.zeros(vocab, grad_out.shape[1], dtype=torch.float64).index_add_(0, t[ok], x.abs()) * abs(s)
    return total, size, torch.bincount(t[ok], minlength=vocab)


def _check(got, total, size, count, old=None):
    """A sum of m binary32 terms in any order is off by at most (m - 1) u (sum of magnitudes) to first order, u = 2^-24; the
    product with the scale adds one u of its value, the sum with the old value one of its own.  The second-order terms are
    below a hundredth of that for the m < 2^17 used here; values below 2^-126 do not occur."""
    u = 2.0 ** -24
    bound = (count.double()[:, None] + 1) * u * size * 1.01
    want = total
    if old is not None:
        want = total + old.double()
        bound = bound + u * (want.abs() + bound) * 1.01
        untouched = count == 0
        assert torch.equal(got[untouched].view(torch.int32), old[untouched].view(torch.int32))
    else:
        assert torch.equal(got[count == 0].view(torch.int32), torch.zeros_like(got[count == 0]).view(torch.int32))
    err = (got.double() - want).abs()
    assert (err <= bound).all(), float((err - bound).max())


CASES = [(1, 1, 1, "uniform"), (1, 9, 650, "uniform"), (5, 3, 33, "same"), (63, 40, 70, "padded"), (128, 300, 513, "text"),
         (128, 10, 4, "same"), (129, 7, 260, "text"), (129, 500, 1, "padded"), (700, 33_278, 650, "text"), (1000, 50, 31, "none"),
         (4095, 16, 129, "uniform"), (4096, 70_000, 64, "text"), (4097, 511, 300, "text"), (4097, 512, 300, "padded"),
         (9000, 3, 40, "uniform"), (20_003, 1 << 18, 24, "text"), (30_000, 17, 1026, "same"), (70_000, 5000, 8, "text"),
         (540_001, 60_000, 3, "text")]


@pytest.mark.parametrize("n,vocab,dim,kind", CASES)
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(n, vocab, dim, kind, accumulate):
    dtype = TYPES[(n + dim) % 3]
    itype = torch.int32 if n % 2 else torch.int64
    scale = [1.0, -0.3][dim % 2]
    _, grad_out = _matrix(n, dim, dtype, 6)
    tokens = _tokens(n, vocab, itype, 7, kind)
    _, table = _matrix(vocab, dim, torch.float32, 8)
    old = table.cpu().clone()
    _gradient(grad_out, tokens.cuda(), table, scale=scale, accumulate=accumulate)
    total, size, count = _expected_gradient(grad_out.cpu(), tokens, vocab, -1, scale)
    _check(table.cpu(), total, size, count, old if accumulate else None)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 128, 129, 3000, 6000])
def test_gradient_sums_of_whole_numbers_are_exact(dtype, n):
    """Whole numbers whose sums stay below 2^24 have no rounding in any order: every row equal, padding and strides included."""
    vocab, dim, padding = 97, 141, 5
    g = torch.Generator().manual_seed(n)
    buf = torch.full((1 + n * (dim + 3),), float("nan"), dtype=dtype)
    buf[1:].view(n, dim + 3)[:, :dim] = torch.randint(-8, 9, (n, dim), generator=g).to(dtype)
    buf = buf.cuda()
    grad_out = buf[1:].view(n, dim + 3)[:, :dim]
    tokens = _tokens(n, vocab, torch.int64, 9, "padded")
    tokens[::5] = padding
    grad_out[(tokens == padding).cuda()] = float("nan")        # a masked place may hold anything
    grad_out[(tokens == -1).cuda()] = float("inf")
    for accumulate in (False, True):
        tbuf = torch.full((3 + vocab * (dim + 2),), 2.0, device="cuda")
        table = tbuf[3:].view(vocab, dim + 2)[:, :dim]
        _gradient(grad_out, tokens.cuda(), table, padding=padding, scale=4.0, accumulate=accumulate)
        ok = (tokens >= 0) & (tokens < vocab) & (tokens != padding)
        want = torch.zeros(vocab, dim, dtype=torch.float64)
        want.index_add_(0, tokens[ok], grad_out.cpu().double()[ok])
        want = want * 4 + (2.0 if accumulate else 0.0)
        assert torch.equal(table.cpu().double(), want)
        got = tbuf.cpu()
        assert (got[3:].view(vocab, dim + 2)[:, dim:] == 2.0).all() and (got[:3] == 2.0).all()


@pytest.mark.parametrize("dim", [1, 2, 3, 4, 5, 7, 8, 9, 11, 255, 257, 259, 511, 513, 519, 2049])
@pytest.mark.parametrize("dtype", TYPES)
def test_ends_of_rows(dtype, dim):
    """Rows that end at any place of a 16-byte access or of a wavefront's columns, strides between them: whole numbers, so that
    every sum is exact, and what lies between the rows is as it was."""
    vocab = 23
    for n in (40, 1500, 4500):
        g = torch.Generator().manual_seed(dim)
        whole = torch.randint(-8, 9, (n, dim), generator=g)
        buf = torch.full((1 + n * (dim + 1),), float("nan"), dtype=dtype)
        buf[1:].view(n, dim + 1)[:, :dim] = whole.to(dtype)
        buf = buf.cuda()
        tokens = _tokens(n, vocab, torch.int32, dim, "padded")
        ok = (tokens >= 0) & (tokens < vocab)
        sums = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, tokens[ok].long(), whole[ok].double())
        for accumulate in (False, True):
            tbuf = torch.full((1 + vocab * (dim + 2),), 3.0, device="cuda")
            _gradient(buf[1:].view(n, dim + 1)[:, :dim], tokens.cuda(), tbuf[1:].view(vocab, dim + 2)[:, :dim], accumulate=accumulate)
            got = tbuf.cpu()
            assert torch.equal(got[1:].view(vocab, dim + 2)[:, :dim].double(), sums + (3.0 if accumulate else 0.0)), (n, accumulate)
            assert (got[1:].view(vocab, dim + 2)[:, dim:] == 3.0).all() and got[0] == 3.0
    out = torch.full((1 + 40 * (dim + 2),), 5.0, dtype=dtype, device="cuda")
    rows = out[1:].view(40, dim + 2)
    B.gravac_embedding_lookup(buf[1:].view(n, dim + 1)[:vocab, :dim], tokens[:40].cuda(), rows[:, :dim])
    want = torch.where(ok[:40, None], whole[tokens[:40].long().clamp(0, vocab - 1)], 0)
    assert torch.equal(rows[:, :dim].cpu().long(), want) and (rows[:, dim:] == 5.0).all() and out[0] == 5.0


@pytest.mark.parametrize("n,vocab", [(8192, 700), (8193, 3), (131_073, 9000), (200_003, 4000), (524_288, 70), (524_289, 1 << 19)])
def test_gradient_of_many_tokens_is_exact(n, vocab):
    """Whole numbers up to 8 in magnitude: sums of at most 2^20 of them are exact."""
    dim = 12
    g = torch.Generator().manual_seed(n)
    whole = torch.randint(-8, 9, (n, dim), generator=g)
    tokens = _tokens(n, vocab, torch.int64, 3, "text")
    table = torch.full((vocab, dim), float("nan"), device="cuda")
    _gradient(whole.to(torch.bfloat16).cuda(), tokens.cuda(), table)
    assert torch.equal(table.cpu().double(), torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, tokens, whole.double()))


def test_gradient_of_no_tokens():
    table = torch.ones(10, 6, device="cuda")
    none, tokens = torch.empty(0, 6, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    _gradient(none, tokens, table, accumulate=True)
    assert (table == 1).all()
    _gradient(none, tokens, table)
    assert torch.equal(table.cpu().view(torch.int32), torch.zeros(10, 6, dtype=torch.int32))


def test_gradient_does_not_depend_on_scheduling_or_on_the_workspace():
    n, vocab, dim = 30_000, 2000, 300
    _, grad_out = _matrix(n, dim, torch.float32, 10)
    tokens = _tokens(n, vocab, torch.int32, 11).cuda()
    size = B.gravac_embedding_gradient_workspace_bytes(n, vocab, dim)
    first = None
    for fill in (0, 255, 1):
        ws = torch.full((size,), fill, dtype=torch.uint8, device="cuda")
        table = torch.empty(vocab, dim, device="cuda")
        _gradient(grad_out, tokens, table, ws=ws)
        got = table.cpu()
        first = got if first is None else first
        assert torch.equal(got.view(torch.int32), first.view(torch.int32))


def test_gradient_is_the_derivative_of_the_lookup():
    """<lookup(E), W> is linear in E: its differences along D are <lookup(D), W> = <gradient(W), D>, both in 64 bits."""
    n, vocab, dim = 5000, 400, 96
    _, D = _matrix(vocab, dim, torch.float32, 12)
    _, W = _matrix(n, dim, torch.float32, 13)
    tokens = _tokens(n, vocab, torch.int64, 14, "padded").cuda()
    out = torch.empty(n, dim, device="cuda")
    B.gravac_embedding_lookup(D, tokens, out, scale=0.7)
    table = torch.empty(vocab, dim, device="cuda")
    _gradient(W, tokens, table, scale=0.7)
    a, b = float((out.double() * W.double()).sum()), float((table.double() * D.double()).sum())
    # each term of the first sum is off by u, each entry of the second by (terms of its row + 1) u
    t = tokens.cpu()
    most = int(torch.bincount(t[(t >= 0) & (t < vocab)]).max())
    bound = (most + 3) * 2.0 ** -24 * float((out.double() * W.double()).abs().sum())
    assert abs(a - b) <= bound


def test_gradient_behind_32_bits():
    vocab, dim = 600_001, 4096
    table = torch.zeros(vocab, dim, device="cuda")
    rows = [0, 524_287, 524_288, 600_000]
    for n in (4, 400):
        tokens = torch.tensor((rows * 100)[:n], dtype=torch.int64, device="cuda")
        grad_out = torch.ones(n, dim, dtype=torch.bfloat16, device="cuda")
        _gradient(grad_out, tokens, table, accumulate=True)
    assert (table[rows] == 101).all()
    assert float(table[::8].double().sum() + table[rows[1:2]].double().sum()) == 101.0 * dim * 4   # rows 0, 524288, 600000 and 524287


@pytest.mark.parametrize("n", [100, 3000, 10_000])
def test_captured_and_replayed_on_a_side_stream(n):
    """The calls on another stream than the default, recorded once and replayed with new inputs, the program's own work
    between the replays; every replay against the eager result."""
    vocab, dim = 700, 130
    tokens = torch.zeros(n, dtype=torch.int64, device="cuda")
    grad_out = torch.zeros(n, dim, device="cuda")
    table, rows = torch.zeros(vocab, dim, device="cuda"), torch.zeros(n, dim, device="cuda")
    weights = torch.randn(vocab, dim, generator=torch.Generator().manual_seed(1)).cuda()
    ws = torch.empty(B.gravac_embedding_gradient_workspace_bytes(n, vocab, dim), dtype=torch.uint8, device="cuda")

    def calls():
        B.gravac_embedding_lookup(weights, tokens, rows)
        _gradient(grad_out, tokens, table, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        t = _tokens(n, vocab, torch.int64, 20 + i, "padded" if i % 2 else "text")
        tokens.copy_(t)
        grad_out.copy_(_matrix(n, dim, torch.float32, 30 + i)[1])
        graph.replay()
        torch.cuda.synchronize()
        want_rows, want = torch.empty_like(rows), torch.empty_like(table)
        B.gravac_embedding_lookup(weights, tokens, want_rows)
        _gradient(grad_out, tokens, want)
        assert torch.equal(rows, want_rows) and torch.equal(table, want)
        total, size, count = _expected_gradient(grad_out.cpu(), t, vocab, -1, 1.0)
        _check(table.cpu(), total, size, count)
        table.fill_(float("nan"))


def test_binding_refuses():
    table, tokens, out = torch.zeros(4, 6, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, 6, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        B.gravac_embedding_lookup(table.cpu(), tokens, out)
    with pytest.raises(ValueError):
        B.gravac_embedding_lookup(table.t(), tokens, out)
    with pytest.raises(ValueError):
        B.gravac_embedding_lookup(table, tokens[:2], out)
    with pytest.raises(ValueError):
        B.gravac_embedding_lookup(table, tokens.float(), out)
    with pytest.raises(TypeError):
        B.gravac_embedding_lookup(table.double(), tokens, out)
    with pytest.raises(TypeError):
        B.gravac_embedding_gradient(out, tokens, table.half(), workspace=ws)
    with pytest.raises(ValueError):
        B.gravac_embedding_gradient(out[:2], tokens, table, workspace=ws)
    with pytest.raises(B.GravacError) as e:
        B.gravac_embedding_gradient(out, tokens, table, workspace=ws[:100])
    assert e.value.code == B.ERR_WORKSPACE
    with pytest.raises(B.GravacError):
        B.gravac_embedding_gradient(out[:1].expand(3, 6), tokens, table, workspace=ws)     # rows one over the other


def _wide_rows(dim, dtype):
    """How many rows of a table a workgroup looks after (those that no token names), and how many workgroups share one group of
    them, for more than 1024 tokens and a table without gaps: the sizes at which the last group is whole, or is not."""
    n = 16 // torch.empty((), dtype=dtype).element_size()
    slabs = -(-dim // (64 * n))
    return max(1, min(64, 65536 // dim)), -(-slabs // min(slabs, 8))


WIDE = [(2052, torch.float32), (2560, torch.float32), (4096, torch.float32), (4100, torch.float32), (8192, torch.bfloat16), (5120, torch.float16),
        (40_000, torch.float32)]


@pytest.mark.parametrize("dim,dtype", WIDE)
def test_gradient_of_wide_rows(dim, dtype):
    """Whole numbers, rows of several workgroups' columns, any number of blocks of rows, the last one whole or not."""
    n = 1100
    rows, columns = _wide_rows(dim, dtype)
    g = torch.Generator().manual_seed(dim)
    whole = torch.randint(-8, 9, (n, dim), generator=g).to(dtype)
    grad_out = whole.cuda()
    for blocks in range(2 * columns, 3 * columns + 1):
        for vocab in {rows * blocks, max(rows * blocks - 3, rows * (blocks - 1) + 1)}:
            tokens = _tokens(n, vocab, torch.int32, blocks, "padded")
            tokens[tokens % 5 == 2] = -1                    # rows that no token names
            ok = (tokens >= 0) & (tokens < vocab)
            table = torch.full((vocab + 2, dim), 3.0, device="cuda")     # two rows behind it
            _gradient(grad_out, tokens.cuda(), table[:vocab])
            want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, tokens[ok].long(), whole[ok].double())
            assert torch.equal(table[:vocab].cpu().double(), want), (blocks, vocab)
            assert (table[vocab:] == 3.0).all()


@pytest.mark.parametrize("dim,dtype", [(2560, torch.float32), (4096, torch.float32), (8192, torch.bfloat16)])
def test_gradient_of_wide_rows_takes_as_long_for_any_number_of_blocks(dim, dtype):
    """A table one block of rows larger costs no more than that block: workgroups that have no block end at once."""
    n = 2000
    rows, columns = _wide_rows(dim, dtype)
    grad_out = torch.zeros(n, dim, dtype=dtype, device="cuda")
    tokens = _tokens(n, 100, torch.int64, 1, "text").cuda()
    took = []
    for blocks in (40 * columns, 40 * columns + 1):
        table = torch.empty(rows * blocks, dim, device="cuda")
        ws = torch.empty(B.gravac_embedding_gradient_workspace_bytes(n, *table.shape), dtype=torch.uint8, device="cuda")
        times = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            _gradient(grad_out, tokens, table, ws=ws)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        took.append(min(times))
    print(dim, dtype, "ms with whole groups of blocks and with one more: %.3f %.3f" % tuple(took))
    assert took[1] < 2 * took[0] + 0.5, took      # (a loop over 2^32 elements takes ten milliseconds and more)


def test_rows_of_two_buffers_that_lie_between_each_other():
    """Two matrices in the columns of one buffer share no element, whatever their spans do: equal strides and one twice the other."""
    vocab, dim, n = 40, 30, 80
    buf = torch.full((2 * vocab * 100,), 7.0, device="cuda")
    table, out = buf.view(vocab, 200)[:, 10:10 + dim], buf.view(n, 100)[:, 50:50 + dim]       # rows 200 and 100 apart
    weights = torch.randn(vocab, dim, generator=torch.Generator().manual_seed(1))
    table.copy_(weights)
    tokens = _tokens(n, vocab, torch.int64, 2, "padded")
    B.gravac_embedding_lookup(table, tokens.cuda(), out, scale=2.0)
    want = _expected_lookup(weights, tokens, 2.0, torch.float32)
    assert torch.equal(out.cpu(), want) and torch.equal(table.cpu(), weights)
    with pytest.raises(B.GravacError) as e:
        B.gravac_embedding_lookup(table, tokens.cuda(), buf.view(n, 100)[:, 39:39 + dim])
    assert e.value.code == B.ERR_INVALID_ARG
    # the gradient: both rows 100 apart
    grad_out, sums = buf.view(n, 100)[:, :dim], buf.view(n, 100)[:vocab, dim:2 * dim]
    grad_out.copy_(want)
    for kw in ({}, {"accumulate": True}):
        sums.fill_(1.0)
        _gradient(grad_out, tokens.cuda(), sums, **kw)
        total, size, count = _expected_gradient(want, tokens, vocab, -1, 1.0)
        _check(sums.cpu(), total, size, count, torch.ones(vocab, dim) if kw else None)
        assert torch.equal(grad_out.cpu(), want)
    with pytest.raises(B.GravacError) as e:
        _gradient(grad_out, tokens.cuda(), buf.view(n, 100)[:vocab, dim - 1:2 * dim - 1])
    assert e.value.code == B.ERR_INVALID_ARG
