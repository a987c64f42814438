"""The grouped products (ecgemm_sgemm_grouped, ecgemm_sgemm_grouped_depth, ecgemm_sgemm_adapters) against the same sums in
64 bits, at the sizes and contents where they can go wrong.

How far an element may be off, derived: with S = sum over k of |a_k| |b_k| for that element,
  * FP16 mode: a pair misses its value by 2^-23 of it, both operands 2^-22 together; the product left out is at most
    2^-11 2^-11 = 2^-22: 2^-21 S.  The residual is a multiple of 2^-24 at the finest, and 2^11 times what it stands for: however
    small a value, the pair may miss it by half of 2^-24 2^-11, 2^-36, which meets the other operand's value: 2^-36 times the
    sum of |a_k| and of |b_k| (and that power of two less for an operand that is scaled before the split).  BF16 mode: three
    terms hold 24 bits, the products left out are below 3 2^-24: less than 2^-21 S again.
  * the matrix unit adds 16 products to an accumulator at a time and drops what lies below 2^-25 of the largest addend, and
    rounds: at most (16 2^-25 + 2^-24) S for each 16 of the depth and each of the two accumulators, which do not both reach S:
    2^-11 S is the other one's, counted as one step more.
  * the merge, alpha, beta and the last rounding: 4 2^-24 (S |alpha| + |beta| |C|).
All operands lie in a field of NaN (leading dimensions, what is before and behind them), so that a value read from outside
would show in the result; all results in a field of one value, so that a value written outside would."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

MODES = ["fp16", "bf16"]


def _ec():
    import paper_2203_03341_amd as ec
    return ec


def _mode(mode):
    ec = _ec()
    return ec.MODE_FP16_SPLIT if mode == "fp16" else ec.MODE_BF16_FULL


@pytest.fixture(scope="module")
def handle():
    import torch
    h = _ec().Handle()
    h.set_stream(torch.cuda.current_stream().cuda_stream)
    yield h
    torch.cuda.synchronize()
    h.destroy()


class Field:
    """`count` column-major rows x cols matrices with leading dimension ld, in a field of `fill`"""

    def __init__(self, rows, cols, pad=0, count=1, gap=0, fill=float("nan"), values=None, wide=False, gen=None, scale=1.0, offset=5):
        import torch
        self.rows, self.cols, self.ld, self.count = rows, cols, max(1, rows + pad), count
        self.stride = self.ld * max(cols, 1) + gap
        self.fill, self.at = fill, 64 + offset
        self.store = torch.full((self.at + self.stride * count + 64,), fill, dtype=torch.float32, device="cuda")
        if values is None and gen is not None:
            values = torch.randn((count, cols, rows), generator=gen, device="cuda", dtype=torch.float64) * scale
            if wide:
                values *= torch.exp2(torch.randint(-40, 21, (count, cols, 1), generator=gen, device="cuda").double())
            values = values.float()
        if values is not None:
            self.view().copy_(values)

    def view(self):
        """(count, cols, rows): [g, j, i] is element (i, j) of matrix g"""
        return self.store.as_strided((self.count, self.cols, self.rows), (self.stride, self.ld, 1), self.at)

    def ptr(self):
        return self.store.data_ptr() + 4 * self.at

    def matrix(self, trans, g=0):
        """op of matrix g in 64 bits, (rows of op, columns of op)"""
        v = self.view()[g].double()
        return v if trans == "T" else v.t()


def _offsets(sizes, start=0):
    import torch
    return torch.tensor(np.concatenate([[start], start + np.cumsum(sizes)]), dtype=torch.int64, device="cuda")


def _allowed(a, b, mode, alpha, beta, before, scaling=(0, 0)):
    """a: M x depth, b: depth x N, in 64 bits"""
    import math
    S, depth = a.abs() @ b.abs(), a.shape[1]
    if mode == "fp16":
        S = S + 2.0 ** 21 * (2.0 ** (-36 - scaling[0]) * b.abs().sum(0)[None, :] + 2.0 ** (-36 - scaling[1]) * a.abs().sum(1)[:, None])
    step = 16 * 2.0 ** -25 + 2.0 ** -24
    bound = (2.0 ** -21 + (math.ceil(depth / 16) + 1) * step) * abs(alpha) * S + 4 * 2.0 ** -24 * abs(alpha) * S
    return bound + (4 * 2.0 ** -24 * abs(beta) * before.abs() if beta else 0.0) + 1e-37


def _ops(trans):
    ec = _ec()
    return {"N": ec.OP_N, "T": ec.OP_T}[trans]


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _run_columns(handle, trans, mode, M, K, sizes, start=0, behind=0, alpha=1.0, beta=0.0, pad=(0, 0, 0), wide=False, seed=1, offset=5,
                 shared=False, scaling=(0, 0)):
    """One call, checked element by element; returns C's field."""
    import torch
    ec, gen = _ec(), _gen(seed)
    N = start + sum(sizes) + behind
    groups = len(sizes)
    a_shape = (M, K) if trans[0] == "N" else (K, M)
    b_shape = (K, N) if trans[1] == "N" else (N, K)
    A = Field(*a_shape, pad=pad[0], count=1 if shared else groups, gap=pad[0], gen=gen, scale=0.5, offset=offset)
    B = Field(*b_shape, pad=pad[1], gen=gen, wide=wide and trans[1] == "N", offset=offset)
    C = Field(M, N, pad=pad[2], fill=7.0, offset=offset)
    if beta:
        C.view().copy_(torch.randn((1, N, M), generator=gen, device="cuda"))
    # what no group holds is never read
    outside = [*range(start), *range(start + sum(sizes), N)]
    b_cols = B.view()[0] if trans[1] == "N" else B.view()[0].t()
    if outside:
        b_cols[outside] = float("nan")
    before = C.store.clone()
    offs = _offsets(sizes, start)
    handle.sgemm_grouped(_ops(trans[0]), _ops(trans[1]), groups, M, N, K, alpha, A.ptr(), A.ld, 0 if shared else A.stride, B.ptr(), B.ld, offs,
                         beta, C.ptr(), C.ld, _mode(mode))
    torch.cuda.synchronize()
    want = before.clone()
    expected = want.as_strided((N, M), (C.ld, 1), C.at)
    got = C.view()[0]
    at = start
    for g, n in enumerate(sizes):
        if n:
            a, b = A.matrix(trans[0], 0 if shared else g), B.matrix(trans[1])[:, at:at + n]
            c_in = expected[at:at + n].t().double()
            exact = alpha * (a @ b) + (beta * c_in if beta else 0.0)
            allowed = _allowed(a, b, mode, alpha, beta, c_in, scaling)
            off = (got[at:at + n].t().double() - exact).abs()
            assert bool((off <= allowed).all()), (trans, mode, M, K, g, n, float((off / allowed).max()))
            expected[at:at + n] = got[at:at + n]
        at += n
    assert torch.equal(C.store, want)       # nothing else was written
    return C


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("trans", ["TN", "NN", "TT", "NT"])
def test_columns_in_every_storage_order(handle, trans, mode):
    _run_columns(handle, trans, mode, 200, 96, [37, 0, 1, 128, 129, 0, 260], start=3, behind=11, pad=(3, 1, 5))
    _run_columns(handle, trans, mode, 384, 512, [256, 128, 384], alpha=1.5, beta=-0.5)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 31, 32, 33, 63, 64, 65, 127, 129, 192, 257, 515])
def test_columns_at_every_kind_of_depth(handle, mode, K):
    for trans in ("TN", "NT"):
        _run_columns(handle, trans, mode, 130, K, [5, 150, 64], behind=2, seed=K, pad=(1, 2, 0))


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 63, 64, 127, 128, 131, 258])
def test_columns_with_few_rows_and_odd_ones(handle, M):
    for trans in ("TN", "NN", "TT"):
        for mode in MODES:
            _run_columns(handle, trans, mode, M, 70, [1, 2, 3, 129], seed=M)


@pytest.mark.parametrize("sizes", [[0], [1], [0, 0, 0], [1] * 40, [0, 0, 300, 0], [513, 1, 0, 2], [128] * 9])
def test_columns_in_groups_of_every_size(handle, sizes):
    for mode in MODES:
        _run_columns(handle, "TN", mode, 140, 130, sizes, start=1, behind=1)
    _run_columns(handle, "NT", "fp16", 140, 130, sizes, start=1, behind=1)


def test_columns_of_any_magnitude_in_bf16_mode(handle):
    _run_columns(handle, "TN", "bf16", 150, 300, [40, 200], wide=True)


def test_columns_many_groups_and_tiles(handle):
    rng = np.random.RandomState(3)
    _run_columns(handle, "TN", "fp16", 40, 33, list(rng.randint(0, 4, 2500)))         # several launches
    _run_columns(handle, "TN", "fp16", 700, 150, list(rng.randint(0, 900, 30)))       # several tiles for every block
    _run_columns(handle, "NN", "bf16", 640, 150, list(rng.randint(0, 900, 30)), beta=1.0)


def test_columns_shared_matrix_and_scaling(handle):
    _run_columns(handle, "TN", "fp16", 130, 100, [60, 70], shared=True)
    handle.set_scaling(6, -3)
    try:
        for mode in MODES:
            _run_columns(handle, "TN", mode, 130, 100, [60, 70], alpha=0.5, beta=2.0, scaling=(6, -3))
            _run_columns(handle, "NT", mode, 130, 300, [60, 70], scaling=(6, -3))
            _run_depth(handle, "NT", mode, 130, 70, [5, 300], scaling=(6, -3))
    finally:
        handle.set_scaling(0, 0)


def _run_depth(handle, trans, mode, M, N, sizes, start=0, behind=0, alpha=1.0, beta=0.0, pad=(0, 0, 0), wide=False, seed=1, offset=5,
               scaling=(0, 0)):
    import torch
    gen = _gen(seed)
    K = start + sum(sizes) + behind
    groups = len(sizes)
    a_shape = (M, K) if trans[0] == "N" else (K, M)
    b_shape = (K, N) if trans[1] == "N" else (N, K)
    A = Field(*a_shape, pad=pad[0], gen=gen, wide=wide and trans[0] == "N", offset=offset)
    B = Field(*b_shape, pad=pad[1], gen=gen, offset=offset)
    outside = [*range(start), *range(start + sum(sizes), K)]
    if outside:
        (A.view()[0] if trans[0] == "N" else A.view()[0].t())[outside] = float("nan")
        (B.view()[0] if trans[1] == "T" else B.view()[0].t())[outside] = float("nan")
    C = Field(M, N, pad=pad[2], count=groups, gap=pad[2], fill=7.0, offset=offset)
    if beta:
        C.view().copy_(torch.randn((groups, N, M), generator=gen, device="cuda"))
    before = C.store.clone()
    handle.sgemm_grouped_depth(_ops(trans[0]), _ops(trans[1]), groups, M, N, K, alpha, A.ptr(), A.ld, B.ptr(), B.ld, _offsets(sizes, start),
                               beta, C.ptr(), C.ld, C.stride, _mode(mode))
    torch.cuda.synchronize()
    want = before.clone()
    expected = want.as_strided((groups, N, M), (C.stride, C.ld, 1), C.at)
    at = start
    for g, n in enumerate(sizes):
        c_in = expected[g].t().double()
        a, b = A.matrix(trans[0])[:, at:at + n], B.matrix(trans[1])[at:at + n]
        exact = alpha * (a @ b) + (beta * c_in if beta else 0.0)
        off = (C.view()[g].t().double() - exact).abs()
        allowed = _allowed(a, b, mode, alpha, beta, c_in, scaling)
        assert bool((off <= allowed).all()), (trans, mode, M, N, g, n, float((off / allowed).max()))
        expected[g] = C.view()[g]
        at += n
    assert torch.equal(C.store, want)
    return C


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("trans", ["NT", "NN", "TT", "TN"])
def test_depth_in_every_storage_order(handle, trans, mode):
    _run_depth(handle, trans, mode, 200, 130, [37, 0, 1, 2, 3, 4, 5, 64, 65, 300], start=3, behind=11, pad=(3, 1, 5))
    _run_depth(handle, trans, mode, 384, 256, [128, 512, 0], alpha=1.5, beta=-0.5)


@pytest.mark.parametrize("M,N", [(1, 1), (3, 5), (127, 129), (2, 260), (260, 2), (128, 128)])
def test_depth_with_few_rows_and_columns(handle, M, N):
    for trans in ("NT", "TN", "TT"):
        for mode in MODES:
            _run_depth(handle, trans, mode, M, N, [1, 33, 0, 200], behind=1, seed=M)


def test_depth_many_groups_and_tiles(handle):
    rng = np.random.RandomState(4)
    _run_depth(handle, "NT", "fp16", 20, 30, list(rng.randint(0, 4, 2100)))
    _run_depth(handle, "NT", "bf16", 300, 400, list(rng.randint(0, 200, 60)), beta=1.0, wide=True)


def _run_adapters(handle, mode, M, N, K, rank, sizes, index, adapters, trans="TNTT", start=0, alpha=1.0, beta=0.0, scales=True, pad=0,
                  wide=False, seed=1):
    """trans: of A, B, D, U"""
    import torch
    gen = _gen(seed)

    def operand(rows, cols, t, **more):
        return Field(rows, cols, gen=gen, pad=pad, **more) if t == "N" else Field(cols, rows, gen=gen, pad=pad, **more)

    A = operand(M, K, trans[0], scale=K ** -0.5 if K else 1.0)
    B = operand(K, N, trans[1], wide=wide and trans[1] == "N")
    D = operand(rank, K, trans[2], count=max(adapters, 1), gap=pad, scale=K ** -0.5 if K else 1.0)
    U = operand(M, rank, trans[3], count=max(adapters, 1), gap=pad, scale=max(rank, 1) ** -0.5)
    s = 0.5 + torch.rand(max(adapters, 1), generator=gen, device="cuda")
    H, C = Field(rank, N, pad=pad, fill=7.0), Field(M, N, pad=pad, fill=7.0)
    if beta:
        C.view().copy_(torch.randn((1, N, M), generator=gen, device="cuda"))
    before_c, before_h = C.store.clone(), H.store.clone()
    handle.sgemm_adapters(_ops(trans[0]), _ops(trans[1]), M, N, K, alpha, A.ptr(), A.ld, B.ptr(), B.ld, len(sizes), _offsets(sizes, start),
                          torch.tensor(index, dtype=torch.int32, device="cuda"), adapters, rank, _ops(trans[2]), D.ptr(), D.ld, D.stride,
                          _ops(trans[3]), U.ptr(), U.ld, U.stride, s if scales else None, H.ptr(), H.ld, beta, C.ptr(), C.ld, _mode(mode))
    torch.cuda.synchronize()
    a, b = A.matrix(trans[0]), B.matrix(trans[1])
    c_in = before_c.as_strided((N, M), (C.ld, 1), C.at).t().double()
    exact = alpha * (a @ b) + (beta * c_in if beta else 0.0)
    allowed = _allowed(a, b, mode, alpha, beta, c_in)
    hidden = torch.zeros((rank, N), dtype=torch.float64, device="cuda")
    hidden_allowed = torch.full((rank, N), 1e-37, dtype=torch.float64, device="cuda")
    at = start
    for g, n in enumerate(sizes):
        if n and 0 <= index[g] < adapters and rank:
            d, u = D.matrix(trans[2], index[g]), U.matrix(trans[3], index[g])
            x, factor = b[:, at:at + n], float(s[index[g]]) if scales else 1.0
            hidden[:, at:at + n] = d @ x
            hidden_allowed[:, at:at + n] = _allowed(d, x, mode, 1.0, 0.0, None)
            # (what H is off by goes through U; the sum meets C in one more rounding)
            h = hidden[:, at:at + n]
            exact[:, at:at + n] += factor * (u @ h)
            allowed[:, at:at + n] += (factor * (u.abs() @ hidden_allowed[:, at:at + n]) + _allowed(u, h, mode, factor, 0.0, None)
                                      + 2.0 ** -23 * exact[:, at:at + n].abs())
        at += n
    off = (H.view()[0].t().double() - hidden).abs()
    assert bool((off <= hidden_allowed).all()), ("H", mode, M, N, K, rank, float((off / hidden_allowed).max()))
    off = (C.view()[0].t().double() - exact).abs()
    assert bool((off <= allowed).all()), ("C", mode, M, N, K, rank, float((off / allowed).max()))
    for field, before in ((C, before_c), (H, before_h)):
        field.view().copy_(before.as_strided(field.view().shape, field.view().stride(), field.at))
        assert torch.equal(field.store, before)     # nothing else was written


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("trans", ["TNTT", "NNNN", "TTTN", "NTNT"])
def test_adapters_in_every_storage_order(handle, trans, mode):
    _run_adapters(handle, mode, 200, 190, 150, 12, [30, 1, 0, 100, 40], [1, -1, 0, 2, 1], 3, trans=trans, start=5, pad=3)
    _run_adapters(handle, mode, 256, 256, 128, 16, [128, 128], [0, 1], 2, trans=trans, alpha=1.5, beta=0.5)


@pytest.mark.parametrize("rank", [1, 2, 3, 4, 7, 8, 16, 20, 33, 64, 65, 130])
def test_adapters_of_every_rank(handle, rank):
    for mode in MODES:
        _run_adapters(handle, mode, 140, 75, 260, rank, [1, 1, 2, 40, 9], [3, 0, 1, 2, -1], 4, seed=rank)


@pytest.mark.parametrize("N", [1, 2, 5, 16, 17, 31, 32, 33, 64, 65])
def test_adapters_of_single_tokens(handle, N):
    """A decoding step: a token and an adapter per request."""
    rng = np.random.RandomState(N)
    for mode in MODES:
        _run_adapters(handle, mode, 300, N, 500, 16, [1] * N, list(rng.randint(-1, 6, N)), 6, seed=N)
        _run_adapters(handle, mode, 1024, N, 1024, 8, [1] * N, list(rng.randint(-1, 6, N)), 6, seed=N, beta=1.0)


def test_adapters_where_there_is_nothing(handle):
    for mode in MODES:
        _run_adapters(handle, mode, 100, 50, 60, 8, [], [], 2)                      # no groups
        _run_adapters(handle, mode, 100, 50, 60, 8, [20, 30], [0, 1], 0)            # no adapters
        _run_adapters(handle, mode, 100, 50, 60, 0, [20, 30], [0, 1], 2)            # no rank
        _run_adapters(handle, mode, 100, 50, 60, 8, [20, 30], [7, -3], 2)           # none that exists
        _run_adapters(handle, mode, 100, 50, 60, 8, [20, 30], [1, 0], 2, alpha=0.0, beta=1.0)
        _run_adapters(handle, mode, 100, 50, 60, 8, [20, 30], [1, 0], 2, scales=False)
        _run_adapters(handle, mode, 100, 50, 0, 8, [20, 30], [1, 0], 2, beta=1.0)   # no depth
    _run_adapters(handle, "bf16", 140, 200, 300, 16, [150, 40], [1, 0], 2, wide=True)


def test_columns_without_depth_or_alpha(handle):
    """C <- beta C in the groups' columns, and A and B are not read."""
    import torch
    ec = _ec()
    for K, alpha in ((0, 1.0), (40, 0.0)):
        for beta in (0.0, 0.5):
            C = Field(30, 20, fill=7.0, values=torch.randn((1, 20, 30), device="cuda"))
            want = C.view().clone()
            want[0, 3:15] = want[0, 3:15] * beta
            handle.sgemm_grouped(ec.OP_T, ec.OP_N, 2, 30, 20, K, alpha, None, 0, 0, None, 0, _offsets([5, 7], 3), beta, C.ptr(), C.ld,
                                 ec.MODE_FP16_SPLIT)
            torch.cuda.synchronize()
            assert torch.equal(C.view(), want)
            C = Field(30, 20, count=2, fill=7.0, values=torch.randn((2, 20, 30), device="cuda"))
            want = C.view() * beta
            handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, 2, 30, 20, K, alpha, None, 0, None, 0, _offsets([5, 7], 3), beta, C.ptr(), C.ld,
                                       C.stride, ec.MODE_BF16_FULL)
            torch.cuda.synchronize()
            assert torch.equal(C.view(), want)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("trans", ["TN", "NT"])
def test_values_that_are_not_finite_stay_in_their_rows_and_columns(handle, trans, mode):
    """An infinity, a NaN and the largest numbers: what they meet may be infinite or NaN, or saturated in FP16 mode; the rest
    is as without them, bit for bit, also what is added to C."""
    import torch
    ec, gen = _ec(), _gen(9)
    M, N, K, sizes = 300, 400, 200, [150, 250]
    a_shape = (M, K) if trans[0] == "N" else (K, M)
    b_shape = (K, N) if trans[1] == "N" else (N, K)
    A, B = Field(*a_shape, count=2, gen=gen), Field(*b_shape, gen=gen)
    results = []
    for spoilt in (False, True):
        a = A.view() if trans[0] == "T" else A.view().transpose(1, 2)      # [g, m, k]
        b = B.view()[0] if trans[1] == "N" else B.view()[0].t()            # [n, k]
        if spoilt:
            a[0, 17, 33] = float("inf")
            a[1, 290, 7] = float("nan")
            b[260, 100] = 3.0e38
            b[399, 199] = -float("inf")
        C = Field(M, N, values=torch.full((1, N, M), 0.25, device="cuda"), fill=7.0)
        handle.sgemm_grouped(_ops(trans[0]), _ops(trans[1]), 2, M, N, K, 1.0, A.ptr(), A.ld, A.stride, B.ptr(), B.ld, _offsets(sizes), 2.0,
                             C.ptr(), C.ld, _mode(mode))
        torch.cuda.synchronize()
        results.append(C.view()[0].clone())     # [n, m]
    clean, spoilt = results
    touched = torch.zeros_like(clean, dtype=torch.bool)
    touched[:150, 17] = touched[150:, 290] = touched[260] = touched[399] = True
    assert torch.equal(clean[~touched], spoilt[~touched])
    assert not bool(torch.isfinite(spoilt[:150, 17]).any())
    assert bool(torch.isnan(spoilt[150:, 290]).all())
    assert not bool(torch.isfinite(spoilt[399]).any())
    if mode == "fp16":      # saturated, not infinite
        assert bool(torch.isfinite(spoilt[260][torch.arange(M, device="cuda") != 290]).all())


def test_offsets_that_no_program_should_pass(handle):
    """Negative, decreasing and far too large offsets: no answer is promised, but nothing outside C is written."""
    import torch
    ec, gen = _ec(), _gen(2)
    M, N, K = 200, 300, 90
    bad = [[-5, 100, 50, 400], [300, 0, 300, 0], [1 << 40, -(1 << 40), 1 << 62, 0], [0, 300, 0, 300], [299, 299, 1 << 33, 3]]
    for offsets in bad:
        offs = torch.tensor(offsets, dtype=torch.int64, device="cuda")
        A, B, C = Field(K, M, count=3, gen=gen), Field(K, N, gen=gen), Field(M, N, pad=4, fill=7.0)
        handle.sgemm_grouped(ec.OP_T, ec.OP_N, 3, M, N, K, 1.0, A.ptr(), A.ld, A.stride, B.ptr(), B.ld, offs, 0.0, C.ptr(), C.ld,
                             ec.MODE_FP16_SPLIT)
        torch.cuda.synchronize()
        C.view().fill_(7.0)
        assert bool((C.store == 7.0).all())
        X, G, W = Field(M, N, gen=gen), Field(K, N, gen=gen), Field(M, K, count=3, fill=7.0, pad=1)
        handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, 3, M, K, N, 1.0, X.ptr(), X.ld, G.ptr(), G.ld, offs, 0.0, W.ptr(), W.ld, W.stride,
                                   ec.MODE_BF16_FULL)
        torch.cuda.synchronize()
        W.view().fill_(7.0)
        assert bool((W.store == 7.0).all())
        D, U, P, H = Field(K, 8, count=2, gen=gen), Field(8, M, count=2, gen=gen), Field(K, M, gen=gen), Field(8, N, fill=7.0)
        handle.sgemm_adapters(ec.OP_T, ec.OP_N, M, N, K, 1.0, P.ptr(), P.ld, B.ptr(), B.ld, 3, offs,
                              torch.tensor([0, 1 << 30, 1], dtype=torch.int32, device="cuda"), 2, 8, ec.OP_T, D.ptr(), D.ld, D.stride, ec.OP_T,
                              U.ptr(), U.ld, U.stride, None, H.ptr(), H.ld, 0.0, C.ptr(), C.ld, ec.MODE_FP16_SPLIT)
        torch.cuda.synchronize()
        C.view().fill_(7.0), H.view().fill_(7.0)
        assert bool((C.store == 7.0).all()) and bool((H.store == 7.0).all())


def test_equal_calls_give_equal_bits_on_any_stream(handle):
    import torch
    first = _run_columns(handle, "TN", "fp16", 300, 700, [100, 5, 300], seed=5).store.clone()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = _ec().Handle()
    other.set_stream(stream.cuda_stream)
    with torch.cuda.stream(stream):
        again = _run_columns(other, "TN", "fp16", 300, 700, [100, 5, 300], seed=5).store.clone()
    torch.cuda.synchronize()
    other.destroy()
    assert torch.equal(first, again)


def test_captured_calls_replay_with_the_offsets_of_the_day():
    """A graph of a layer of experts, forward and backward, and of a projection with adapters."""
    import torch
    ec, gen = _ec(), _gen(6)
    E, T, K, M, R = 4, 300, 160, 190, 8
    x, g = torch.randn((T, K), generator=gen, device="cuda"), torch.randn((T, M), generator=gen, device="cuda")
    W = torch.randn((E, M, K), generator=gen, device="cuda")
    D, U = torch.randn((3, R, K), generator=gen, device="cuda"), torch.randn((3, M, R), generator=gen, device="cuda")
    offs, index = torch.zeros(E + 1, dtype=torch.int64, device="cuda"), torch.zeros(E, dtype=torch.int32, device="cuda")
    outs = [torch.zeros((T, M), device="cuda"), torch.zeros((T, K), device="cuda"), torch.zeros((E, M, K), device="cuda"),
            torch.zeros((T, M), device="cuda"), torch.zeros((T, R), device="cuda")]

    def calls(h, y, dx, dw, z, hid):
        h.sgemm_grouped(ec.OP_T, ec.OP_N, E, M, T, K, 1.0, W, K, M * K, x, K, offs, 0.0, y, M, ec.MODE_FP16_SPLIT)
        h.sgemm_grouped(ec.OP_N, ec.OP_N, E, K, T, M, 1.0, W, K, M * K, g, M, offs, 0.0, dx, K, ec.MODE_FP16_SPLIT)
        h.sgemm_grouped_depth(ec.OP_N, ec.OP_T, E, K, M, T, 1.0, x, K, g, M, offs, 0.0, dw, K, M * K, ec.MODE_BF16_FULL)
        h.sgemm_adapters(ec.OP_T, ec.OP_N, M, T, K, 1.0, W, K, x, K, E, offs, index, 3, R, ec.OP_T, D, K, R * K, ec.OP_T, U, R, M * R, None,
                         hid, R, 0.0, z, M, ec.MODE_FP16_SPLIT)

    captured, eager = ec.Handle(), ec.Handle()
    eager.set_stream(torch.cuda.current_stream().cuda_stream)
    nbytes = max(256, captured.workspace_size(ec.OP_T, ec.OP_N, M, T, K, ec.MODE_FP16_SPLIT))
    workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    captured.set_workspace(workspace, nbytes)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.set_stream(torch.cuda.current_stream().cuda_stream)
        calls(captured, *outs)
    for sizes, ids in (([100, 0, 150, 50], [0, 1, 2, 0]), ([1, 1, 1, 1], [2, -1, 0, 0]), ([0, 0, 0, 300], [1, 1, 1, 1]), ([75] * 4, [0, 5, 2, 1])):
        offs.copy_(_offsets(sizes)), index.copy_(torch.tensor(ids, dtype=torch.int32, device="cuda"))
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = [torch.zeros_like(o) for o in outs]
        calls(eager, *want)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)
    captured.destroy(), eager.destroy()


def test_a_layer_of_experts_forward_and_backward(handle):
    """y = W2[e] relu(W1[e] x): the program's calls one after the other, against autograd in 64 bits and against differences."""
    import torch
    ec, gen = _ec(), _gen(11)
    E, T, K, F, M = 5, 230, 96, 160, 72
    sizes, mode = [60, 0, 1, 100, 69], ec.MODE_FP16_SPLIT
    offs = _offsets(sizes)
    x = torch.randn((T, K), generator=gen, device="cuda")
    W1, W2 = torch.randn((E, F, K), generator=gen, device="cuda") / K ** 0.5, torch.randn((E, M, F), generator=gen, device="cuda") / F ** 0.5
    gy = torch.randn((T, M), generator=gen, device="cuda")

    def up(W, rows, width, out):    # rows of `width` times W[e]^T
        n = W.shape[1]
        handle.sgemm_grouped(ec.OP_T, ec.OP_N, E, n, T, width, 1.0, W, width, n * width, rows, width, offs, 0.0, out, n, mode)
        return out

    def back(W, rows, out):
        n, width = W.shape[1], W.shape[2]
        handle.sgemm_grouped(ec.OP_N, ec.OP_N, E, width, T, n, 1.0, W, width, n * width, rows, n, offs, 0.0, out, width, mode)
        return out

    def weights(rows, grads, out):
        n, width = grads.shape[1], rows.shape[1]
        handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, E, width, n, T, 1.0, rows, width, grads, n, offs, 0.0, out, width, n * width, mode)
        return out

    h = up(W1, x, K, torch.empty((T, F), device="cuda"))
    a = h.relu()
    y = up(W2, a, F, torch.empty((T, M), device="cuda"))
    ga = back(W2, gy, torch.empty((T, F), device="cuda"))
    gW2 = weights(a, gy, torch.empty_like(W2))
    gh = ga * (h > 0)
    gx = back(W1, gh, torch.empty((T, K), device="cuda"))
    gW1 = weights(x, gh, torch.empty_like(W1))
    torch.cuda.synchronize()

    def layer(x, W1, W2):
        out, at = [], 0
        for e, n in enumerate(sizes):
            out.append((x[at:at + n] @ W1[e].t()).relu() @ W2[e].t())
            at += n
        return torch.cat(out)

    leaves = [v.cpu().double().requires_grad_() for v in (x, W1, W2)]
    want = layer(*leaves)
    grads = torch.autograd.grad((want * gy.cpu().double()).sum(), leaves)
    for got, ref in zip((y, gx, gW1, gW2), (want, *grads)):
        off = float((got.cpu().double() - ref.detach()).norm() / ref.detach().norm())
        # two products after each other, each off by at most 2^-21 + 11 (16 2^-25 + 2^-24) of S; in the 2-norm S is at most
        # sqrt(depth) times the result's for independent values, and errors of independent elements add up as their root
        # does: 2 sqrt(160) 6.4e-6 / sqrt(160)
        assert off < 1.3e-5, off
    # One difference along a random direction, in 64 bits: <grad, d> against (f(v + d) - f(v - d)) / 2.  f is linear in each leaf
    # between relu's corners.  A value h that passes its corner between h - e and h + e adds e relu' on one side only, so the
    # difference misses its part of <grad, d> by at most |df/da| |e|, added up over those that do.
    # <grad, d> itself is off by what the gradient is, at most 1.3e-5 of its 2-norm as above, times d's: an independent random
    # direction meets it with 1 / sqrt(count) of that, for which ten standard deviations are allowed.
    directions = torch.Generator().manual_seed(14)
    for i, got in ((0, gx), (1, gW1), (2, gW2)):
        v = [l.detach() for l in leaves]
        d = 1e-7 * torch.randn(v[i].shape, generator=directions, dtype=torch.float64)
        moved = {sign: [u + sign * d if k == i else u for k, u in enumerate(v)] for sign in (1.0, -1.0)}
        f = {sign: (layer(*moved[sign]) * gy.cpu().double()).sum() for sign in moved}
        difference, along = float(f[1.0] - f[-1.0]) / 2, float((got.cpu().double() * d).sum())
        corners, at = 0.0, 0
        for e, n in enumerate(sizes):
            h_up, h_down = (moved[sign][0][at:at + n] @ moved[sign][1][e].t() for sign in (1.0, -1.0))
            passing = (h_up > 0) != (h_down > 0)
            corners += float(((gy[at:at + n].cpu().double() @ moved[1.0][2][e]).abs() * (h_up - h_down).abs() / 2)[passing].sum())
            at += n
        off = 10 * 1.3e-5 * float(got.double().norm()) * float(d.norm()) / d.numel() ** 0.5
        assert abs(difference - along) <= off + corners + 1e-10, (i, difference, along, off, corners)


def test_adapters_forward_and_backward(handle):
    """A projection with an adapter per task: forward, and the gradients of the input and of the adapters."""
    import torch
    ec, gen = _ec(), _gen(12)
    T, K, M, R = 210, 120, 88, 8
    sizes, mode = [50, 60, 100], ec.MODE_FP16_SPLIT
    offs, index = _offsets(sizes), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    x, gy = torch.randn((T, K), generator=gen, device="cuda"), torch.randn((T, M), generator=gen, device="cuda")
    W = torch.randn((M, K), generator=gen, device="cuda") / K ** 0.5
    D, U = torch.randn((3, R, K), generator=gen, device="cuda") / K ** 0.5, torch.randn((3, M, R), generator=gen, device="cuda") / R ** 0.5
    scale = 2.0
    scales = torch.full((3,), scale, device="cuda")
    y, H = torch.empty((T, M), device="cuda"), torch.empty((T, R), device="cuda")
    gx, gH = torch.empty((T, K), device="cuda"), torch.empty((T, R), device="cuda")
    gD, gU = torch.empty_like(D), torch.empty_like(U)
    handle.sgemm_adapters(ec.OP_T, ec.OP_N, M, T, K, 1.0, W, K, x, K, 3, offs, index, 3, R, ec.OP_T, D, K, R * K, ec.OP_T, U, R, M * R, scales,
                          H, R, 0.0, y, M, mode)
    handle.sgemm_adapters(ec.OP_N, ec.OP_N, K, T, M, 1.0, W, K, gy, M, 3, offs, index, 3, R, ec.OP_N, U, R, M * R, ec.OP_N, D, K, R * K, scales,
                          gH, R, 0.0, gx, K, mode)
    handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, 3, K, R, T, scale, x, K, gH, R, offs, 0.0, gD, K, R * K, mode)
    handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, 3, R, M, T, scale, H, R, gy, M, offs, 0.0, gU, R, M * R, mode)
    torch.cuda.synchronize()
    leaves = [v.cpu().double().requires_grad_() for v in (x, D, U)]
    out, at = [], 0
    for e, n in enumerate(sizes):
        rows = leaves[0][at:at + n]
        out.append(rows @ W.cpu().double().t() + scale * (rows @ leaves[1][e].t()) @ leaves[2][e].t())
        at += n
    want = torch.cat(out)
    grads = torch.autograd.grad((want * gy.cpu().double()).sum(), leaves)
    for got, ref in zip((y, gx, gD, gU), (want, *grads)):
        off = float((got.cpu().double() - ref.detach()).norm() / ref.detach().norm())
        assert off < 1.3e-5, off    # as for the layer of experts


def test_refusals(handle):
    """Whatever is wrong with a call: the status, which argument, and nothing enqueued."""
    import torch
    ec = _ec()
    t = torch.zeros(4096, device="cuda")
    offs, index = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    names = {"sgemm_grouped": "transA transB groups M N K alpha A lda strideA B ldb offsets beta C ldc mode",
             "sgemm_grouped_depth": "transA transB groups M N K alpha A lda B ldb offsets beta C ldc strideC mode",
             "sgemm_adapters": "transA transB M N K alpha A lda B ldb groups offsets index adapters rank transD D ldd strideD transU U ldu strideU "
                               "scales H ldh beta C ldc mode"}
    sound = dict(transA=ec.OP_T, transB=ec.OP_N, groups=3, M=8, N=8, K=8, alpha=1.0, A=t, lda=8, strideA=64, B=t[1024:], ldb=8, offsets=offs,
                 beta=0.0, C=t[2048:], ldc=8, strideC=64, mode=ec.MODE_FP16_SPLIT, index=index, adapters=2, rank=4, transD=ec.OP_T, D=t, ldd=8,
                 strideD=32, transU=ec.OP_T, U=t, ldu=4, strideU=32, scales=None, H=t[2560:], ldh=4)
    wrong = {name: [dict(transA=2), dict(transB=-1), dict(M=-1), dict(N=-1), dict(K=-1), dict(groups=-1), dict(A=None), dict(lda=7), dict(B=None),
                    dict(ldb=7), dict(C=None), dict(ldc=7), dict(offsets=None), dict(offsets=offs.data_ptr() + 4), dict(mode=11), dict(mode=-1),
                    dict(M=1 << 31), dict(N=1 << 31), dict(K=1 << 31, lda=1 << 31, ldb=1 << 31), dict(groups=1 << 31)] for name in names}
    wrong["sgemm_grouped"] += [dict(strideA=-1), dict(lda=(1 << 21) + 1), dict(ldb=(1 << 21) + 1)]
    wrong["sgemm_grouped_depth"] += [dict(strideC=63), dict(ldc=1 << 62)]
    wrong["sgemm_adapters"] += [dict(transD=3), dict(transU=3), dict(rank=-1), dict(rank=1025), dict(adapters=-1), dict(adapters=1 << 31),
                                dict(index=None), dict(index=index.data_ptr() + 2), dict(D=None), dict(ldd=7), dict(strideD=-1), dict(U=None),
                                dict(ldu=3), dict(strideU=-1), dict(H=None), dict(ldh=3)]
    alias = {"ldc": ["ldc", "strideC"]}
    for name, order in names.items():
        order = order.split()
        for change in wrong[name]:
            with pytest.raises(ec.EcgemmError) as err:
                getattr(handle, name)(*[{**sound, **change}[k] for k in order])
            key = next(iter(change))
            positions = [order.index(k) + 2 for k in alias.get(key, [key]) if k in order]
            assert err.value.status == ec.ERR_INVALID_ARG and err.value.argument in positions, (name, change, err.value, err.value.argument)
        for mode in (ec.MODE_AUTO, ec.MODE_FP32_MFMA, ec.MODE_FP16_MARKIDIS):
            with pytest.raises(ec.EcgemmError) as err:
                getattr(handle, name)(*[{**sound, "mode": mode}[k] for k in order])
            assert err.value.status == ec.ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert bool((t == 0).all())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("trans", ["TNTT", "NNNN", "TNTN", "TTTT"])
@pytest.mark.parametrize("N", [24, 150, 600])
def test_an_adapter_that_is_not_finite_stays_with_its_columns(handle, trans, mode, N):
    """What an adapter of one request holds does not reach the others, whichever kernels make the product."""
    import torch
    ec, gen = _ec(), _gen(13)
    M, K, R = 300, 200, 12
    sizes, index = [N // 6, N // 3, N // 6, N // 6], [0, 1, 2, 0]

    def operand(rows, cols, t, **more):
        return Field(rows, cols, gen=gen, **more) if t == "N" else Field(cols, rows, gen=gen, **more)

    A, B = operand(M, K, trans[0]), operand(K, N, trans[1])
    D, U = operand(R, K, trans[2], count=3), operand(M, R, trans[3], count=3)
    results = []
    for spoilt in (False, True):
        if spoilt:
            U.view()[1].fill_(float("nan"))
            D.view()[2][3, 5] = float("inf")
        H, C = Field(R, N, fill=7.0), Field(M, N, values=torch.full((1, N, M), 0.25, device="cuda"), fill=7.0)
        handle.sgemm_adapters(_ops(trans[0]), _ops(trans[1]), M, N, K, 1.0, A.ptr(), A.ld, B.ptr(), B.ld, 4, _offsets(sizes, 2),
                              torch.tensor(index, dtype=torch.int32, device="cuda"), 3, R, _ops(trans[2]), D.ptr(), D.ld, D.stride,
                              _ops(trans[3]), U.ptr(), U.ld, U.stride, None, H.ptr(), H.ld, 2.0, C.ptr(), C.ld, _mode(mode))
        torch.cuda.synchronize()
        results.append((C.view()[0].clone(), H.view()[0].clone()))
    at = np.cumsum([2, *sizes])
    others = [*range(at[0]), *range(at[0], at[1]), *range(at[3], N)]
    (clean, h_clean), (bad, h_bad) = results
    assert torch.equal(clean[others], bad[others]) and torch.equal(h_clean[others], h_bad[others])
    assert bool(torch.isnan(bad[at[1]:at[2]]).all())
    assert torch.equal(h_clean[at[1]:at[2]], h_bad[at[1]:at[2]])
    assert not bool(torch.isfinite(bad[at[2]:at[3]]).all(dim=1).any())


@pytest.mark.parametrize("mode", MODES)
def test_deep_products_of_few_tiles_are_added_up_from_slices(handle, mode):
    """Slices of the depth through the workspace: every storage order, ragged depths, nothing in some groups, and a caller's
    workspace of the promised size."""
    import torch
    ec = _ec()
    workspace = torch.full((ec.GROUPED_WORKSPACE_BYTES // 4 + 64,), 3.0, device="cuda")
    for trans in ("TN", "NT", "NN", "TT"):
        _run_columns(handle, trans, mode, 200, 2500, [140, 0, 300], start=1, behind=3, alpha=1.5, beta=-0.5, pad=(1, 2, 3))
        _run_depth(handle, trans, mode, 130, 90, [2000, 3, 0, 5001], behind=7, alpha=1.5, beta=-0.5, pad=(1, 2, 3))
    own = ec.Handle()
    own.set_stream(torch.cuda.current_stream().cuda_stream)
    own.set_workspace(workspace, ec.GROUPED_WORKSPACE_BYTES)
    _run_depth(own, "NT", mode, 1000, 1000, [9000])
    _run_depth(own, "NT", mode, 100, 100, [40000])
    _run_columns(own, "TN", mode, 128, 4100, [256])
    torch.cuda.synchronize()
    assert bool((workspace[ec.GROUPED_WORKSPACE_BYTES // 4:] == 3.0).all())
    own.set_workspace(workspace, 256)
    with pytest.raises(ec.EcgemmError) as err:
        _run_depth(own, "NT", mode, 100, 100, [40000])
    assert err.value.status == ec.ERR_ALLOC
    own.destroy()


@pytest.mark.parametrize("mode", MODES)
def test_values_that_are_not_finite_in_slices_and_few_columns(handle, mode):
    """A NaN in one slice of the depth, and with few columns, stays in its row; the rest is as without it, bit for bit."""
    import torch
    ec, gen = _ec(), _gen(21)
    for M, N, K in ((150, 260, 3000), (150, 9, 300)):
        A, B = Field(K, M, count=2, gen=gen), Field(K, N, gen=gen)
        sizes, results = [N // 2, N - N // 2], []
        for spoilt in (False, True):
            if spoilt:
                A.view()[1, 77, K - 5] = float("nan")
            C = Field(M, N, values=torch.full((1, N, M), 0.25, device="cuda"), fill=7.0)
            handle.sgemm_grouped(ec.OP_T, ec.OP_N, 2, M, N, K, 1.0, A.ptr(), A.ld, A.stride, B.ptr(), B.ld, _offsets(sizes), 2.0, C.ptr(), C.ld,
                                 _mode(mode))
            torch.cuda.synchronize()
            results.append(C.view()[0].clone())
        touched = torch.zeros_like(results[0], dtype=torch.bool)
        touched[N // 2:, 77] = True
        assert torch.equal(results[0][~touched], results[1][~touched]) and bool(torch.isnan(results[1][touched]).all())


def test_adapters_of_the_largest_rank_and_through_the_workspace(handle):
    """Ranks beyond a few passes; and the way that takes the handle's workspace refuses a small one before it writes anything."""
    import torch
    ec = _ec()
    for mode in MODES:
        _run_adapters(handle, mode, 70, 40, 90, 1024, [20, 20], [1, 0], 2)
        _run_adapters(handle, mode, 130, 300, 90, 1024, [200, 90], [1, 0], 2, trans="NNTN")
    own = ec.Handle()
    own.set_stream(torch.cuda.current_stream().cuda_stream)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    own.set_workspace(small, 256)
    H, C = torch.full((2000, 8), 7.0, device="cuda"), torch.full((2000, 2000), 7.0, device="cuda")
    x, W, D = (torch.randn((2000, 7000), device="cuda") for _ in range(3))
    with pytest.raises(ec.EcgemmError) as err:      # (too deep for one launch)
        own.sgemm_adapters(ec.OP_T, ec.OP_N, 2000, 2000, 7000, 1.0, W, 7000, x, 7000, 2, _offsets([1000, 1000]), _offsets([1]).int(), 1, 8, ec.OP_T, D,
                           7000, 0, ec.OP_T, D, 8, 0, None, H, 8, 0.0, C, 2000, ec.MODE_FP16_SPLIT)
    assert err.value.status == ec.ERR_ALLOC
    torch.cuda.synchronize()
    assert bool((H == 7.0).all()) and bool((C == 7.0).all())
    own.destroy()


def test_an_infinite_alpha_does_not_meet_what_is_not_there(handle):
    """No depth: C <- beta C, whatever alpha is."""
    import torch
    ec = _ec()
    for N, M in ((20, 30), (600, 300)):
        C = Field(M, N, fill=7.0, values=torch.randn((1, N, M), device="cuda"))
        want = C.view() * 0.5
        handle.sgemm_grouped(ec.OP_T, ec.OP_N, 1, M, N, 0, float("inf"), None, 0, 0, None, 0, _offsets([N]), 0.5, C.ptr(), C.ld, ec.MODE_FP16_SPLIT)
        torch.cuda.synchronize()
        assert torch.equal(C.view(), want)
    X, G, C = Field(30, 5), Field(20, 5), Field(30, 20, count=2, fill=7.0, values=torch.randn((2, 20, 30), device="cuda"))
    want = C.view()[1] * 0.5
    handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, 2, 30, 20, 5, float("inf"), X.ptr(), X.ld, G.ptr(), G.ld, _offsets([5, 0]), 0.5, C.ptr(), C.ld,
                               C.stride, ec.MODE_BF16_FULL)
    torch.cuda.synchronize()
    assert torch.equal(C.view()[1], want)


@pytest.mark.parametrize("trans", ["NNNN", "TNTT", "TNTN", "NTNT", "TTTT"])
def test_adapters_of_single_tokens_in_more_than_one_pass(handle, trans):
    """Decoding steps of more requests than a pass of the narrow kernel holds, in the storage orders of forward and backward: the
    adapters of a pass must not be those of the next one."""
    rng = np.random.RandomState(31)
    for M, K, N, R in ((1826, 3000, 40, 48), (300, 900, 64, 16), (258, 700, 130, 12)):
        for mode in MODES:
            _run_adapters(handle, mode, M, N, K, R, [1] * (N - 3), list(rng.randint(-1, 5, N - 3)), 5, trans=trans, start=1, seed=N)


@pytest.mark.parametrize("M", [4, 8, 12, 48, 60, 62, 64, 68, 100])
def test_few_columns_with_contiguous_rows_of_every_number(handle, M):
    for trans in ("NN", "NT"):
        _run_columns(handle, trans, "fp16", M, 200, [1, 3, 17, 33, 2], start=1, behind=1, pad=(1, 0, 2), seed=M)


@pytest.mark.parametrize("trans", ["NT", "NN", "TT", "TN"])
def test_shallow_groups_of_the_depth(handle, trans):
    """Groups a few deep, few and many rows and columns, each way of adding to C; and as deep as one of them happens to be."""
    for mode in MODES:
        _run_depth(handle, trans, mode, 260, 130, [1, 0, 2, 16, 17, 3, 5, 0], start=2, behind=3, pad=(1, 2, 3))
        _run_depth(handle, trans, mode, 256, 128, [1, 4, 33, 0, 0, 0, 1, 1], alpha=1.5, beta=-0.5)
        _run_depth(handle, trans, mode, 7, 300, [40, 100, 0], alpha=-1.0, beta=1.0, pad=(2, 0, 1))
        _run_depth(handle, trans, mode, 300, 5, [64, 20, 9], pad=(0, 1, 0))
        _run_depth(handle, trans, mode, 64, 64, [1] * 70)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("M", [33, 34, 35, 61, 129, 130, 131, 133, 254, 255, 257, 387])
def test_contiguous_rows_of_every_remainder(handle, M, mode):
    """The last rows of a tile are fewer than a load takes: they come with earlier ones, and none is written twice or skipped."""
    _run_columns(handle, "NT", mode, M, 333, [1, 7, 30, 2], alpha=1.5, beta=-0.5, pad=(1, 0, 2), seed=M)
    _run_columns(handle, "NN", mode, M, 520, [150, 129, 200], start=1, behind=2, alpha=1.5, beta=-0.5, pad=(0, 1, 0), seed=M)
    _run_columns(handle, "NT", mode, M, 65, [M, 129, 0, 200], pad=(2, 3, 0), seed=M)
    _run_depth(handle, "NT", mode, M, M + 1, [500, 129, 64, 0, 321], alpha=1.5, beta=1.0, pad=(1, 1, 1), seed=M)
    _run_adapters(handle, mode, M, 24, 200, 8, [3, 9, 12], [1, 0, 1], 2, trans="NNNN", beta=0.5)
    _run_adapters(handle, mode, M, 300, 200, 8, [100, 41, 159], [1, 0, 1], 2, trans="NNNN", beta=0.5)


@pytest.mark.parametrize("mode", MODES)
def test_values_that_are_not_finite_in_the_last_contiguous_rows(handle, mode):
    import torch
    ec = _ec()
    for M, N, K in [(131, 200, 192), (131, 12, 192), (387, 300, 65), (61, 20, 64)]:
        A, B = torch.randn((K, M), device="cuda"), torch.randn((N, K), device="cuda")
        A[K // 2, M - 1] = float("inf")
        B[3, 5] = float("nan")
        C = torch.full((N, M), 7.0, device="cuda")
        handle.sgemm_grouped(ec.OP_N, ec.OP_N, 1, M, N, K, 1.0, A.data_ptr(), M, 0, B.data_ptr(), K, _offsets([N]), 0.0, C.data_ptr(), M,
                             _mode(mode))
        exact = (B.double().cpu() @ A.double().cpu()).cuda()
        mask = exact.isfinite()
        assert torch.equal(C.isfinite(), mask)      # (an infinity may come out as a NaN: its parts meet others of either sign)
        a, b = A.clone(), B.clone()
        a[K // 2, M - 1] = 0.0
        b[3, 5] = 0.0
        allowed = _allowed(a.t().double(), b.t().double(), mode, 1.0, 0.0, None).t()
        assert bool(((C.double() - exact).abs()[mask] <= allowed[mask]).all())


@pytest.mark.parametrize("M", [2001, 2050, 2051])
def test_adapters_in_tiles_with_contiguous_rows_of_every_remainder(handle, M):
    _run_adapters(handle, "fp16", M, 1100, 150, 20, [500, 1, 599], [1, 0, 1], 2, trans="NNNN", beta=0.5, pad=1)
    _run_adapters(handle, "bf16", M, 1100, 150, 20, [500, 1, 599], [1, 0, 1], 2, trans="NNTN", pad=1)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("trans", ["NT", "NN", "TT", "TN"])
def test_shallow_groups_keep_to_themselves(handle, trans, mode):
    """What is not finite in one group's tokens reaches that group's C only, and there the row or column it belongs to."""
    import torch
    gen, M, N, sizes = _gen(3), 200, 140, [3, 0, 5, 1, 18, 2]
    K, starts = sum(sizes), np.concatenate([[0], np.cumsum(sizes)])
    A = Field(*((M, K) if trans[0] == "N" else (K, M)), gen=gen)
    B = Field(*((K, N) if trans[1] == "N" else (N, K)), gen=gen)
    results = []
    for spoilt in (False, True):
        a = A.view()[0] if trans[0] == "N" else A.view()[0].t()     # [k, m]
        b = B.view()[0].t() if trans[1] == "N" else B.view()[0]     # [k, n]
        if spoilt:
            a[starts[2] + 1, 7] = float("inf")
            a[starts[4] + 17, 199] = float("nan")
            b[starts[2], 139] = -float("inf")
            b[starts[5], 0] = float("nan")
        C = Field(M, N, count=len(sizes), gap=3, fill=7.0)
        handle.sgemm_grouped_depth(_ops(trans[0]), _ops(trans[1]), len(sizes), M, N, K, 1.0, A.ptr(), A.ld, B.ptr(), B.ld, _offsets(sizes),
                                   0.0, C.ptr(), C.ld, C.stride, _mode(mode))
        torch.cuda.synchronize()
        results.append(C.view().clone())     # [g, n, m]
    clean, spoilt = results
    touched = torch.zeros_like(clean, dtype=torch.bool)
    touched[2, :, 7] = touched[2, 139] = touched[4, :, 199] = touched[5, 0] = True
    assert torch.equal(clean[~touched], spoilt[~touched])
    assert not bool(torch.isfinite(spoilt[touched]).any())


def test_one_group_of_the_most_columns_there_can_be(handle):
    """Rounding its columns up to whole tiles passes 32 bits.  Every element is written, and none before or behind C."""
    import torch
    ec, N, guard = _ec(), (1 << 31) - 1, 1024
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB of GPU memory")
    A = torch.full((1,), 2.0, device="cuda")
    B, C = (torch.full((N + 2 * guard,), v, device="cuda") for v in (1.5, 7.0))
    ends = {0: 5.0, 1: -1.0, 126: 4.0, 128: 9.0, N // 2: 0.25, N - 128: 6.0, N - 2: 8.0, N - 1: -3.0}
    for j, v in ends.items():
        B[guard + j] = v
    handle.sgemm_grouped(ec.OP_N, ec.OP_N, 1, 1, N, 1, 1.0, A, 1, 1, B[guard:], 1, _offsets([N]), 0.0, C[guard:], 1, ec.MODE_FP16_SPLIT)
    torch.cuda.synchronize()
    for j, v in ends.items():       # products of a few bits: exact in either mode
        assert float(C[guard + j]) == 2.0 * v, j
        C[guard + j] = 3.0
    assert bool((C[:guard] == 7.0).all()) and bool((C[guard + N:] == 7.0).all())
    step = 1 << 28
    assert all(bool((C[guard + at:min(guard + at + step, guard + N)] == 3.0).all()) for at in range(0, N, step))


def test_calls_that_no_single_launch_holds(handle):
    """More groups than one launch of the kernel that suits their size: another one makes them."""
    import torch
    ec, gen = _ec(), _gen(41)
    # 131072 groups of a column each, one matrix for all
    G, M, K = 131072, 1024, 16
    A, x = torch.randn((M, K), generator=gen, device="cuda"), torch.randn((G, K), generator=gen, device="cuda")
    y = torch.full((G, M), 7.0, device="cuda")
    offs = torch.arange(G + 1, device="cuda")
    handle.sgemm_grouped(ec.OP_T, ec.OP_N, G, M, G, K, 1.0, A, K, 0, x, K, offs, 0.0, y, M, ec.MODE_FP16_SPLIT)
    torch.cuda.synchronize()
    for at in range(0, G, 16384):
        rows = slice(at, at + 16384)
        allowed = _allowed(x[rows].double(), A.double().t().contiguous(), "fp16", 1.0, 0.0, None)
        assert bool(((y[rows].double() - x[rows].double() @ A.double().t().contiguous()).abs() <= allowed).all())
    # 2^24 gradients of one value
    G = 1 << 24
    x, g, c = torch.randn(G, generator=gen, device="cuda"), torch.randn(G, generator=gen, device="cuda"), torch.full((G,), 7.0, device="cuda")
    handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, G, 1, 1, G, 1.0, x, 1, g, 1, torch.arange(G + 1, device="cuda"), 0.0, c, 1, 1, ec.MODE_BF16_FULL)
    torch.cuda.synchronize()
    exact = x.double() * g.double()     # one product: what _allowed gives for a depth of 1
    assert bool(((c.double() - exact).abs() <= (2.0 ** -21 + 2 * (16 * 2.0 ** -25 + 2.0 ** -24) + 4 * 2.0 ** -24) * exact.abs() + 1e-37).all())


def test_adapters_of_more_requests_than_a_launch_holds(handle):
    import torch
    ec, gen = _ec(), _gen(42)
    G, M, K, R = 131072, 8, 16, 1024
    x, W = torch.randn((G, K), generator=gen, device="cuda"), torch.randn((M, K), generator=gen, device="cuda")
    D, U = torch.randn((2, R, K), generator=gen, device="cuda"), torch.randn((2, M, R), generator=gen, device="cuda") / 32
    index = torch.randint(-1, 2, (G,), generator=gen, device="cuda", dtype=torch.int32)
    y, H = torch.full((G, M), 7.0, device="cuda"), torch.full((G, R), 7.0, device="cuda")
    handle.sgemm_adapters(ec.OP_T, ec.OP_N, M, G, K, 1.0, W, K, x, K, G, torch.arange(G + 1, device="cuda"), index, 2, R, ec.OP_T, D, K, R * K,
                          ec.OP_T, U, R, M * R, None, H, R, 0.0, y, M, ec.MODE_FP16_SPLIT)
    torch.cuda.synchronize()
    for a in (-1, 0, 1):
        rows = (index == a).nonzero()[:, 0]
        b, h = x[rows].double(), H[rows]
        exact, allowed = b @ W.double().t().contiguous(), _allowed(b, W.double().t().contiguous(), "fp16", 1.0, 0.0, None)
        if a < 0:
            assert bool((h == 0).all())
        else:
            d, u = D[a].double().t().contiguous(), U[a].double().t().contiguous()
            want, h_allowed = b @ d, _allowed(b, d, "fp16", 1.0, 0.0, None)
            assert bool(((h.double() - want).abs() <= h_allowed).all())
            exact = exact + want @ u
            allowed = allowed + h_allowed @ u.abs() + _allowed(want, u, "fp16", 1.0, 0.0, None) + 2.0 ** -23 * exact.abs()
        assert bool(((y[rows].double() - exact).abs() <= allowed).all())


def test_adapters_that_no_launch_holds_are_refused_before_anything_is_written(handle):
    import torch
    ec = _ec()
    t = torch.zeros(4096, device="cuda")
    offs, index = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")

    def call(M, N, alpha):
        handle.sgemm_adapters(ec.OP_T, ec.OP_N, M, N, 8, alpha, t, 8, t, 8, 3, offs, index, 2, 4, ec.OP_T, t, 8, 32, ec.OP_T, t, 4, 32, None,
                              t[2048:], 4, 0.0, t[3000:], M, ec.MODE_FP16_SPLIT)

    for position, sizes in ((5, (8, 1 << 30, 1.0)), (4, ((1 << 31) - 1, 1024, 0.0))):
        with pytest.raises(ec.EcgemmError) as err:
            call(*sizes)
        assert err.value.status == ec.ERR_INVALID_ARG and err.value.argument == position
    torch.cuda.synchronize()
    assert bool((t == 0).all())


@pytest.mark.parametrize("mode", MODES)
def test_the_last_of_several_launches_takes_its_groups_for_as_deep_as_they_are(handle, mode):
    """1025 groups are two launches, the second one of a single group.  A hundred deep each, they are cut into no slices, so that a
    caller's workspace of any size does; two thousand deep, the last one is, and a workspace too small for it is refused before
    anything is written."""
    import torch
    ec, G = _ec(), 1025
    own = ec.Handle()
    own.set_stream(torch.cuda.current_stream().cuda_stream)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    own.set_workspace(small, 256)
    _run_depth(own, "NT", mode, 65, 66, [100] * G)
    M, N, K = 65, 66, 2048 * G
    A, B, C = torch.ones((K, M), device="cuda"), torch.ones((K, N), device="cuda"), torch.full((G, N, M), 7.0, device="cuda")
    args = (ec.OP_N, ec.OP_T, G, M, N, K, 1.0, A, M, B, N, torch.arange(G + 1, device="cuda") * 2048, 1.0, C, M, M * N, _mode(mode))
    with pytest.raises(ec.EcgemmError) as err:
        own.sgemm_grouped_depth(*args)
    assert err.value.status == ec.ERR_ALLOC
    torch.cuda.synchronize()
    assert bool((C == 7.0).all())
    own.set_workspace(None, 0)
    own.sgemm_grouped_depth(*args)
    torch.cuda.synchronize()
    assert bool((C == 2055.0).all())        # (sums of ones: exact)
    own.destroy()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("sizes,index", [([50, 0, 60, 33, 1, 27, 40], [2, 1, 0, -1, 2, 0, 5]), ([5, 70, 3], [0, 0, 0]), ([40, 50], [-1, 3])])
def test_gradients_of_adapters_that_requests_share(handle, mode, sizes, index):
    """Every adapter with a scale of its own, adapters that several requests share, that one has and that none has, requests without
    one, rows of no request: the gradients of the input, of D and of U as the interface says they are made, against autograd in 64
    bits and against differences."""
    import torch
    ec, gen, A, E = _ec(), _gen(51), 4, len(sizes)
    K, M, R, start = 120, 88, 8, 2
    T = start + sum(sizes) + 3
    offs, ids = _offsets(sizes, start), torch.tensor(index, dtype=torch.int32, device="cuda")
    x, gy = torch.randn((T, K), generator=gen, device="cuda"), torch.randn((T, M), generator=gen, device="cuda")
    W = torch.randn((M, K), generator=gen, device="cuda") / K ** 0.5
    D, U = torch.randn((A, R, K), generator=gen, device="cuda") / K ** 0.5, torch.randn((A, M, R), generator=gen, device="cuda") / R ** 0.5
    scales = torch.tensor([0.5, -1.25, 2.0, 3.0], device="cuda")
    y, H = torch.empty((T, M), device="cuda"), torch.empty((T, R), device="cuda")
    gx, gH = torch.empty((T, K), device="cuda"), torch.empty((T, R), device="cuda")
    handle.sgemm_adapters(ec.OP_T, ec.OP_N, M, T, K, 1.0, W, K, x, K, E, offs, ids, A, R, ec.OP_T, D, K, R * K, ec.OP_T, U, R, M * R, scales,
                          H, R, 0.0, y, M, _mode(mode))
    handle.sgemm_adapters(ec.OP_N, ec.OP_N, K, T, M, 1.0, W, K, gy, M, E, offs, ids, A, R, ec.OP_N, U, R, M * R, ec.OP_N, D, K, R * K, scales,
                          gH, R, 0.0, gx, K, _mode(mode))
    of_group_d, of_group_u = torch.empty((E, R, K), device="cuda"), torch.empty((E, M, R), device="cuda")
    handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, E, K, R, T, 1.0, x, K, gH, R, offs, 0.0, of_group_d, K, R * K, _mode(mode))
    handle.sgemm_grouped_depth(ec.OP_N, ec.OP_T, E, R, M, T, 1.0, H, R, gy, M, offs, 0.0, of_group_u, R, M * R, _mode(mode))
    torch.cuda.synchronize()
    gD, gU = torch.zeros_like(D), torch.zeros_like(U)
    for e, a in enumerate(index):
        if 0 <= a < A:
            gD[a] += scales[a] * of_group_d[e]
            gU[a] += scales[a] * of_group_u[e]
    w, s = W.cpu().double(), scales.cpu().double()

    def call(x, D, U):
        out, at = [x[:start] @ w.t()], start
        for n, a in zip(sizes, index):
            rows = x[at:at + n]
            out.append(rows @ w.t() + (s[a] * (rows @ D[a].t()) @ U[a].t() if 0 <= a < A else 0.0))
            at += n
        return torch.cat([*out, x[at:] @ w.t()])

    leaves = [v.cpu().double().requires_grad_() for v in (x, D, U)]
    want, g = call(*leaves), gy.cpu().double()
    grads = torch.autograd.grad((want * g).sum(), leaves, allow_unused=True)
    directions = torch.Generator().manual_seed(52)
    for i, (got, ref) in enumerate(zip((gx, gD, gU), grads)):
        ref, got = torch.zeros_like(leaves[i]) if ref is None else ref, got.cpu().double()
        # two products after each other, as for the layer of experts; a sum of groups adds a rounding of its result for each of them
        assert float((got - ref).norm()) <= (1.3e-5 + len(sizes) * 2.0 ** -24) * float(ref.norm())
        # f is linear in each of its arguments: its difference is <gradient, d> but for the roundings of 64 bits
        d = torch.randn(got.shape, generator=directions, dtype=torch.float64)
        v = [l.detach() for l in leaves]
        difference = float(((call(*[u + d if k == i else u for k, u in enumerate(v)]) - call(*v)) * g).sum())
        rounding = 1e-9 * (1.0 + float(g.norm()) * float(want.detach().norm()))
        assert abs(difference - float((ref * d).sum())) <= rounding
        assert abs(difference - float((got * d).sum())) <= rounding + 1.4e-5 * float(ref.norm()) * float(d.norm())
    assert float((y.cpu().double() - want.detach()).norm()) <= 1.3e-5 * float(want.detach().norm())
    for a in range(A):
        if a not in index:
            assert not bool(gD[a].any()) and not bool(gU[a].any())


@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("trans", ["NT", "NN", "TT", "TN"])
@pytest.mark.parametrize("M,N,groups,deep", [(70, 80, 300, 4800), (64, 200, 150, 9600), (257, 65, 64, 1000)])
def test_one_group_as_deep_as_all_of_them(handle, trans, M, N, groups, deep, positive):
    """Groups that are shallow on average, one of which has all the depth: its sums run along the depth in FP32.  Derived: a
    fused multiply-add for each of n products, each rounded by 2^-24 of a sum that S bounds: n 2^-24 S, and 4 2^-24 S for
    alpha and the rest.  And as close as the library promises of every product: the relative residual against 64 bits at most
    1.25 times that of a naive FP32 product."""
    import torch
    from oracle import gemm
    gen = _gen(61)
    a_shape, b_shape = ((M, deep) if trans[0] == "N" else (deep, M)), ((deep, N) if trans[1] == "N" else (N, deep))
    A, B = Field(*a_shape, gen=gen), Field(*b_shape, gen=gen)
    if positive:
        A.view().abs_(), B.view().abs_()
    C = Field(M, N, count=groups, fill=7.0)
    sizes = [0] * groups
    sizes[groups // 3] = deep
    for mode in MODES:
        handle.sgemm_grouped_depth(_ops(trans[0]), _ops(trans[1]), groups, M, N, deep, 1.5, A.ptr(), A.ld, B.ptr(), B.ld, _offsets(sizes), 0.0,
                                   C.ptr(), C.ld, C.stride, _mode(mode))
        torch.cuda.synchronize()
        a, b, got = A.matrix(trans[0]), B.matrix(trans[1]), C.view()[groups // 3].t()
        exact = 1.5 * (a @ b)
        assert bool(((got.double() - exact).abs() <= (deep + 4) * 2.0 ** -24 * 1.5 * (a.abs() @ b.abs())).all())
        rows, cols = (np.asfortranarray(v.float().cpu().numpy()) for v in (a, b))
        naive = gemm.sgemm_fp32_naive("N", "N", M, N, deep, 1.5, rows, cols)
        assert gemm.relative_residual(exact.cpu().numpy(), got.cpu().numpy()) <= 1.25 * gemm.relative_residual(exact.cpu().numpy(), naive)
        others = [g for g in range(groups) if g != groups // 3]
        assert not bool(C.view()[others].any())


def test_few_columns_of_a_great_depth(handle):
    """The sums of few columns run along the depth in FP32, in eight parts."""
    import torch
    from oracle import gemm
    gen, M, N, K = _gen(62), 4096, 5, 60000
    A, B, C = Field(K, M, gen=gen), Field(K, N, gen=gen), Field(M, N, fill=7.0)
    handle.sgemm_grouped(_ops("T"), _ops("N"), 1, M, N, K, 1.0, A.ptr(), A.ld, 0, B.ptr(), B.ld, _offsets([N]), 0.0, C.ptr(), C.ld, _mode("fp16"))
    torch.cuda.synchronize()
    a, b, got = A.matrix("T"), B.matrix("N"), C.view()[0].t()
    exact = a @ b
    # an eighth of the depth in a row, at most a stretch of 32 more, then eight sums one after the other
    assert bool(((got.double() - exact).abs() <= (K / 8 + 32 + 8 + 4) * 2.0 ** -24 * (a.abs() @ b.abs())).all())
    rows = 40
    naive = gemm.sgemm_fp32_naive("N", "N", rows, N, K, 1.0, *(np.asfortranarray(v.float().cpu().numpy()) for v in (a[:rows], b)))
    want = exact[:rows].cpu().numpy()
    assert gemm.relative_residual(want, got[:rows].cpu().numpy()) <= 1.25 * gemm.relative_residual(want, naive)


def test_a_forced_shape_and_the_timing_switch_leave_groups_alone(handle):
    """Equal bits with and without either; the projection of adapters may be made by ecgemm_sgemm's kernels, which follow both."""
    import torch
    ec = _ec()
    want = [_run_columns(handle, "TN", "fp16", 300, 200, [100, 400]).store.clone(), _run_depth(handle, "NT", "bf16", 300, 200, [100, 400]).store.clone()]
    other = ec.Handle()
    other.set_stream(torch.cuda.current_stream().cuda_stream)
    other.set_timing(True)
    for shape in (ec.SHAPE_256x128_W4, ec.SHAPE_64x64_FUSED, ec.SHAPE_AUTO):
        other.set_shape(shape)
        got = [_run_columns(other, "TN", "fp16", 300, 200, [100, 400]).store, _run_depth(other, "NT", "bf16", 300, 200, [100, 400]).store]
        assert all(torch.equal(g.nan_to_num(), w.nan_to_num()) for g, w in zip(got, want))
        for mode in MODES:
            _run_adapters(other, mode, 140, 200, 300, 16, [150, 40], [1, 0], 2, beta=0.5)
    torch.cuda.synchronize()
    other.destroy()


# more than 128 tiles: projection and adapters in one launch (A and U stored alike, the depth contiguous in B)
_TILES = dict(M=2050, N=1100, K=150)


@pytest.mark.parametrize("mode,rank", [("fp16", 20), ("fp16", 72), ("bf16", 20), ("bf16", 40)])
@pytest.mark.parametrize("trans", ["TNTT", "NNNN", "TNNT", "NNTN"])
def test_adapters_in_tiles(handle, trans, mode, rank):
    """Adapters of a chunk and of more, several of them meeting in a tile, and columns without one."""
    _run_adapters(handle, mode, **_TILES, rank=rank, sizes=[100, 1, 30, 0, 5, 400, 60, 17, 300], index=[2, 0, -1, 1, 3, 1, 7, 2, 0], adapters=4,
                  trans=trans, start=3, alpha=1.5, beta=-0.5, pad=1)
    _run_adapters(handle, mode, 2048, 1152, 128, rank, [128, 300, 724], [1, -1, 0], 2, trans=trans)


@pytest.mark.parametrize("mode,rank", [("fp16", 20), ("fp16", 72), ("bf16", 20), ("bf16", 40)])
@pytest.mark.parametrize("trans", ["TNTT", "NNNN", "TNNT", "NNTN"])
def test_an_adapter_that_is_not_finite_in_tiles(handle, trans, mode, rank):
    """Tiles that hold columns of such adapters, of sound ones and of none are made again for each of them: the others' bits are
    those without it, and C, which is added to, is added once."""
    import torch
    ec, gen = _ec(), _gen(71)
    M, N, K = (_TILES[k] for k in "MNK")
    sizes, index, start = [200, 90, 7, 33, 300, 250, 150], [0, 1, -1, 3, 2, 0, 3], 5

    def operand(rows, cols, t, **more):
        return Field(rows, cols, gen=gen, **more) if t == "N" else Field(cols, rows, gen=gen, **more)

    A, B = operand(M, K, trans[0]), operand(K, N, trans[1])
    D, U = operand(rank, K, trans[2], count=4), operand(M, rank, trans[3], count=4)
    scales = torch.tensor([0.5, 1.5, -2.0, 1.0], device="cuda")
    results = []
    for spoilt in (False, True):
        if spoilt:
            U.view()[1].fill_(float("nan"))
            U.view()[2][rank - 1 if trans[3] == "N" else 1999, 1999 if trans[3] == "N" else rank - 1] = float("inf")
            D.view()[3][3, 5] = float("inf")
        H, C = Field(rank, N, fill=7.0), Field(M, N, values=torch.full((1, N, M), 0.25, device="cuda"), fill=7.0)
        handle.sgemm_adapters(_ops(trans[0]), _ops(trans[1]), M, N, K, 1.0, A.ptr(), A.ld, B.ptr(), B.ld, len(sizes), _offsets(sizes, start),
                              torch.tensor(index, dtype=torch.int32, device="cuda"), 4, rank, _ops(trans[2]), D.ptr(), D.ld, D.stride,
                              _ops(trans[3]), U.ptr(), U.ld, U.stride, scales, H.ptr(), H.ld, 2.0, C.ptr(), C.ld, _mode(mode))
        torch.cuda.synchronize()
        results.append((C.view()[0].clone(), H.view()[0].clone()))
        field = C.store.clone()
        field.as_strided((N, M), (C.ld, 1), C.at).fill_(7.0)
        assert bool((field == 7.0).all())
    (clean, h_clean), (bad, h_bad) = results
    of = torch.full((N,), -1)
    at = start
    for n, a in zip(sizes, index):
        of[at:at + n] = a
        at += n
    of = of.cuda()
    sound = (of == -1) | (of == 0)
    assert bool(torch.isfinite(clean).all()) and torch.equal(clean[sound], bad[sound])
    assert torch.equal(h_clean[of != 3], h_bad[of != 3])
    assert bool(torch.isnan(bad[of == 1]).all())
    others = torch.arange(M, device="cuda") != 1999        # of the one infinite value of U_2: its row alone
    assert torch.equal(clean[of == 2][:, others], bad[of == 2][:, others]) and not bool(torch.isfinite(bad[of == 2][:, 1999]).any())
    assert not bool(torch.isfinite(bad[of == 3]).any())


@pytest.mark.parametrize("trans", ["TN", "TT"])
def test_few_columns_in_blocks_of_two_rows(handle, trans):
    """More than 16 columns to a group and 256 blocks of 32 rows: a block takes that many."""
    rng = np.random.RandomState(81)
    for K in (200, 33):
        _run_columns(handle, trans, "fp16", 261, K, list(rng.randint(17, 32, 32)), start=1, behind=2, alpha=1.5, beta=-0.5, pad=(1, 2, 3), seed=K)
    _run_columns(handle, trans, "bf16", 256, 192, [32, 1, 17, 63, 0, 33, 40, 16] * 4)


@pytest.mark.parametrize("trans", ["TNTT", "TNNT", "NNNN", "NNTN"])
@pytest.mark.parametrize("rank", [17, 20, 64, 100])
def test_adapters_of_many_columns_in_blocks_of_two_rows(handle, trans, rank):
    """H of more than 8160 columns in blocks of 32 of them, adapters meeting within a block."""
    sizes, index = [3000, 1, 2, 29, 0, 1500, 40, 3600], [0, 2, 1, 0, 1, 2, -1, 1]
    _run_adapters(handle, "fp16", 20, 8200, 90, rank, sizes, index, 3, trans=trans, start=7, pad=1, seed=rank)
    _run_adapters(handle, "bf16", 5, 8192, 64, rank, [4096, 4096], [1, 0], 2, trans=trans, beta=0.5, seed=rank)


@pytest.mark.parametrize("trans", ["TNTT", "TTTN"])
def test_adapters_of_few_columns_in_blocks_of_two_rows(handle, trans):
    """A projection of 8161 rows or more and 17 columns or more."""
    rng = np.random.RandomState(82)
    for M, N, K in ((8200, 40, 300), (8161, 17, 65), (8192, 64, 256)):
        _run_adapters(handle, "fp16", M, N, K, 12, [1] * (N - 3) + [2], list(rng.randint(-1, 4, N - 2)), 4, trans=trans, beta=0.5, seed=N)


@pytest.mark.parametrize("mode", MODES)
def test_adapters_whose_projection_is_a_product_of_its_own(handle, mode):
    """C of the adapters first, the projection added by ecgemm_sgemm's kernels: with a pre-scaling, an alpha by which H is not to
    be divided, a great depth, A and U stored differently, and more requests than meet in a tile."""
    import torch
    for alpha, beta in ((2.0 ** -20, 0.0), (2.0 ** 18, 2.0 ** 18)):
        _run_adapters(handle, mode, **_TILES, rank=20, sizes=[500, 1, 590], index=[1, -1, 0], adapters=2, start=3, alpha=alpha, beta=beta)
    _run_adapters(handle, mode, M=2050, N=1100, K=6200, rank=20, sizes=[500, 1, 590], index=[1, -1, 0], adapters=2, beta=1.0, start=3, pad=1)
    _run_adapters(handle, mode, **_TILES, rank=8, sizes=[500, 600], index=[1, 0], adapters=2, trans="NNNT", beta=1.0)
    _run_adapters(handle, mode, **_TILES, rank=8, sizes=[9] * 122, index=[1, 0] * 61, adapters=2, start=1)
    other = _ec().Handle()
    other.set_stream(torch.cuda.current_stream().cuda_stream)
    other.set_scaling(2, 3)
    _run_adapters(other, mode, **_TILES, rank=8, sizes=[500, 600], index=[1, 0], adapters=2, beta=1.0)
    torch.cuda.synchronize()
    other.destroy()


def test_captured_calls_that_use_the_workspace(handle):
    """Slices of the depth and a projection that is split first, in a graph on a caller's workspace, between eager calls of another
    handle: every replay has the bits of the eager call."""
    import torch
    ec, gen = _ec(), _gen(91)
    T, K, M, R, N = 3000, 300, 200, 8, 1024
    x, g = torch.randn((T, K), generator=gen, device="cuda"), torch.randn((T, M), generator=gen, device="cuda")
    W, rows = torch.randn((2048, 7000), generator=gen, device="cuda") / 80, torch.randn((N, 7000), generator=gen, device="cuda")
    D, U = torch.randn((2, R, 7000), generator=gen, device="cuda") / 80, torch.randn((2, 2048, R), generator=gen, device="cuda")
    offs, offs_n, index = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")

    def calls(h, dw, y, hidden):
        h.sgemm_grouped_depth(ec.OP_N, ec.OP_T, 2, K, M, T, 1.0, x, K, g, M, offs, 0.0, dw, K, M * K, ec.MODE_FP16_SPLIT)
        h.sgemm_adapters(ec.OP_T, ec.OP_N, 2048, N, 7000, 1.0, W, 7000, rows, 7000, 2, offs_n, index, 2, R, ec.OP_T, D, 7000, R * 7000, ec.OP_T, U, R,
                         2048 * R, None, hidden, R, 0.0, y, 2048, ec.MODE_BF16_FULL)

    outs = [torch.zeros((2, M, K), device="cuda"), torch.zeros((N, 2048), device="cuda"), torch.zeros((N, R), device="cuda")]
    captured, eager = ec.Handle(), ec.Handle()
    eager.set_stream(torch.cuda.current_stream().cuda_stream)
    nbytes = max(ec.GROUPED_WORKSPACE_BYTES, captured.workspace_size(ec.OP_T, ec.OP_N, 2048, N, 7000, ec.MODE_BF16_FULL))
    workspace = torch.full((nbytes // 4 + 64,), 3.0, device="cuda")
    captured.set_workspace(workspace, nbytes)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.set_stream(torch.cuda.current_stream().cuda_stream)
        calls(captured, *outs)
    for sizes, ids in (([1000, 2000], [0, 1]), ([3000, 0], [1, 1]), ([1, 2], [-1, 0]), ([1500, 1500], [1, -1])):
        offs.copy_(_offsets(sizes)), offs_n.copy_(_offsets([s // 3 for s in sizes])), index.copy_(torch.tensor(ids, dtype=torch.int32, device="cuda"))
        want = [torch.full_like(o, 5.0) for o in outs]
        calls(eager, *want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)
    assert bool((workspace[nbytes // 4:] == 3.0).all())
    captured.destroy(), eager.destroy()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("trans", ["TN", "NN", "TT", "NT"])
def test_scaling_in_every_storage_order(handle, trans, mode):
    """The handle's pre-scaling in tiles, whole and ragged, and in slices of the depth."""
    handle.set_scaling(6, -3)
    try:
        _run_columns(handle, trans, mode, 300, 200, [150, 3, 400], start=1, behind=2, alpha=0.5, beta=2.0, pad=(1, 2, 3), scaling=(6, -3))
        _run_columns(handle, trans, mode, 256, 192, [256, 384], scaling=(6, -3))
        _run_depth(handle, trans, mode, 300, 200, [150, 0, 401], start=1, beta=1.0, pad=(1, 2, 3), scaling=(6, -3))
        _run_depth(handle, trans, mode, 130, 90, [2000, 3, 4001], alpha=1.5, scaling=(6, -3))
    finally:
        handle.set_scaling(0, 0)


def test_columns_in_tiles_of_several_launches(handle):
    """More than 1024 groups, each with a matrix of its own, of more columns than the kernel of few columns takes."""
    rng = np.random.RandomState(101)
    _run_columns(handle, "TN", "fp16", 9, 10, list(rng.randint(60, 260, 1100)), start=2, behind=1, pad=(1, 0, 1))


@pytest.mark.parametrize("trans", ["TN", "NN", "TT", "NT"])
def test_the_largest_leading_dimensions(handle, trans):
    """2^21 from one column to the next, in tiles, with few columns, and in shallow groups."""
    def pads(*rows):
        return tuple((1 << 21) - r for r in rows)

    def stored(rows, cols, t):
        return rows if t == "N" else cols

    M, K = 130, 97
    for mode in MODES:
        N = 140
        _run_columns(handle, trans, mode, M, K, [N], alpha=1.5, pad=(*pads(stored(M, K, trans[0]), stored(K, N, trans[1])), 1))
    N = 19
    _run_columns(handle, trans, "fp16", M, K, [N], pad=(*pads(stored(M, K, trans[0]), stored(K, N, trans[1])), 1))
    M, N = 129, 130
    for sizes in ([200], [5, 9]):
        K = sum(sizes)
        _run_depth(handle, trans, "fp16", M, N, sizes, pad=(*pads(stored(M, K, trans[0]), stored(K, N, trans[1])), 1))


@pytest.mark.parametrize("N", [30, 400])
def test_the_first_half_of_adapters_alone(handle, N):
    """No rows of C: H all the same, and neither A nor U nor C is looked at."""
    import torch
    ec, gen, K, R = _ec(), _gen(111), 90, 12
    x, D = torch.randn((N, K), generator=gen, device="cuda"), torch.randn((2, R, K), generator=gen, device="cuda")
    H, sizes = torch.full((N, R), 7.0, device="cuda"), [N // 2, N // 4]
    handle.sgemm_adapters(ec.OP_T, ec.OP_N, 0, N, K, 1.0, None, 0, x, K, 2, _offsets(sizes), torch.tensor([1, 0], dtype=torch.int32, device="cuda"),
                          2, R, ec.OP_T, D, K, R * K, ec.OP_T, None, 0, 0, None, H, R, 0.0, None, 0, ec.MODE_FP16_SPLIT)
    torch.cuda.synchronize()
    at = 0
    for n, a in zip(sizes, (1, 0)):
        b, d = x[at:at + n].double(), D[a].double().t().contiguous()
        assert bool(((H[at:at + n].double() - b @ d).abs() <= _allowed(b, d, "fp16", 1.0, 0.0, None)).all())
        at += n
    assert not bool(H[at:].any())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("M,N", [(2050, 1100), (300, 600), (300, 24)])
def test_a_scale_that_is_not_finite_stays_with_its_adapter(handle, mode, M, N):
    import torch
    ec, gen, K, R = _ec(), _gen(112), 150, 12
    W, x = torch.randn((M, K), generator=gen, device="cuda"), torch.randn((N, K), generator=gen, device="cuda")
    D, U = torch.randn((3, R, K), generator=gen, device="cuda"), torch.randn((3, M, R), generator=gen, device="cuda")
    sizes, index, results = [N // 4, N // 6, N // 6], [0, 1, 2], []
    for scales in ([0.5, 1.0, 2.0], [0.5, float("nan"), float("inf")]):
        y, H = torch.full((N, M), 0.25, device="cuda"), torch.full((N, R), 7.0, device="cuda")
        handle.sgemm_adapters(ec.OP_T, ec.OP_N, M, N, K, 1.0, W, K, x, K, 3, _offsets(sizes), torch.tensor(index, dtype=torch.int32, device="cuda"),
                              3, R, ec.OP_T, D, K, R * K, ec.OP_T, U, R, M * R, torch.tensor(scales, device="cuda"), H, R, 2.0, y, M, _mode(mode))
        torch.cuda.synchronize()
        results.append((y, H))
    (clean, h_clean), (bad, h_bad) = results
    at = np.cumsum([0, *sizes])
    others = [*range(at[1]), *range(at[3], N)]
    assert torch.equal(h_clean, h_bad) and torch.equal(clean[others], bad[others]) and bool(torch.isfinite(clean).all())
    assert bool(torch.isnan(bad[at[1]:at[2]]).all()) and not bool(torch.isfinite(bad[at[2]:at[3]]).any())
