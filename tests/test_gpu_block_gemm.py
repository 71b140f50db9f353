"""Products of 8-bit matrices against 64 bits: whole numbers exactly, others within a bound derived from the number of additions."""
import numpy as np
import pytest
import torch

from paper_1705_05249_amd import experts as X
from tests import expert_reference as R

pytestmark = pytest.mark.gpu
CODE = {"f32": X.MG_F32, "f16": X.MG_F16, "bf16": X.MG_BF16}
TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def kind_of_scales(pow2, kind="f32"):
    """with sums in FP32: what C in FP32 gets anyway"""
    return (X.MG_SCALES_POW2 if pow2 else X.MG_SCALES_ANY) | (0 if kind == "f32" else X.MG_SUMS_FP32)


def operand(rng, rows, k, square, pow2, whole, ld, start):
    """(bytes with NaN between the rows, scales with NaN behind the rows', values, tensors)"""
    if whole:                                               # small whole numbers and scales with an exact product
        q = R.round_e4m3(rng.integers(-8, 9, (rows, k)).astype(np.float64))
    else:
        q = R.round_e4m3(rng.standard_normal((rows, k)) * np.exp2(rng.integers(-6, 6, (rows, k))))
    tall, across = (-(-rows // 128) if square else rows), -(-k // 128)
    if whole:
        s = np.exp2(rng.integers(-2, 3, (tall, across)).astype(np.float64))
    else:
        s = np.exp2(rng.integers(-9, 4, (tall, across)).astype(np.float64))
        if not pow2:
            s = (s * rng.uniform(1, 2, s.shape)).astype(np.float32).astype(np.float64)
    stored = np.full(start + rows * ld + 32, 0x7F, np.uint8)
    stored[start:start + rows * ld].reshape(rows, ld)[:, :k] = q
    scales = np.full((tall, across + 1), np.nan, np.float32)
    scales[:, :across] = s
    return R.values(q, s, square), torch.tensor(stored).cuda()[start:], torch.tensor(scales).cuda()


def check(m, n, k, layout=X.MG_ROW_MAJOR, kind="f32", a_square=False, b_square=True, pow2=False, whole=False, alpha=1.0, beta=0.0, ld=None, starts=(0, 0, 0),
          ldc=None, workspace=True, seed=0):
    print(m, n, k, layout, kind, a_square, b_square, pow2, whole, alpha, beta, ld, starts, ldc, workspace, flush=True)
    rng = np.random.default_rng(seed + m * 7 + n * 11 + k)
    lda, ldb = ld or (max(k, 1), max(k, 1))
    a, A, SA = operand(rng, m, k, a_square, pow2, whole, lda, starts[0])
    b, B, SB = operand(rng, n, k, b_square, pow2, whole, ldb, starts[1])
    row = layout == X.MG_ROW_MAJOR
    major, minor = (m, n) if row else (n, m)
    ldc = ldc or minor
    old = torch.tensor(np.round(rng.standard_normal((major, ldc)) * 4)).to(TYPE[kind])
    buf = torch.full((starts[2] + major * ldc + 16,), 7.0, dtype=TYPE[kind], device="cuda")
    buf[starts[2]:starts[2] + major * ldc] = (old if beta else torch.full_like(old, float("nan"))).reshape(-1).cuda()
    before = buf.clone()
    need = X.mg_block_gemm_workspace_bytes(m, n, k)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if workspace and need else None
    X.mg_block_gemm(layout, m, n, k, alpha, kind_of_scales(pow2, kind), X.MG_BLOCK_SQUARE if a_square else X.MG_BLOCK_ROW, A, lda, SA, SA.shape[1],
                    X.MG_BLOCK_SQUARE if b_square else X.MG_BLOCK_ROW, B, ldb, SB, SB.shape[1], beta, CODE[kind], buf[starts[2]:], ldc, ws)
    torch.cuda.synchronize()
    got = buf[starts[2]:starts[2] + major * ldc].view(major, ldc)[:, :minor].double().cpu().numpy()
    outside = torch.ones_like(buf, dtype=torch.bool)
    outside[starts[2]:starts[2] + major * ldc].view(major, ldc)[:, :minor] = False
    assert torch.equal(buf[outside].nan_to_num(3.0), before[outside].nan_to_num(3.0)), "written outside C"
    c = old[:, :minor].double().numpy()
    if not row:
        got, c = got.T, c.T
    want, magnitudes = R.product(a, b, alpha, beta, c)
    if whole:
        want = torch.tensor(want).to(TYPE[kind]).double().numpy()
        assert np.array_equal(got, want)
    else:
        bound = R.product_bound(want, magnitudes, k, kind)
        assert R.near(got, want, bound, kind)


SIZES = [(1, 1, 1), (1, 16, 128), (1, 100, 1000), (2, 300, 129), (5, 257, 640), (16, 128, 127), (17, 33, 300), (31, 64, 256), (64, 64, 64), (65, 200, 384),
         (100, 1, 500), (128, 128, 128), (129, 127, 144), (200, 300, 1000), (256, 256, 512), (257, 513, 400), (300, 8, 2064)]


@pytest.mark.parametrize("kind", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("pow2", (False, True))
def test_sizes(kind, pow2):
    for m, n, k in SIZES:
        check(m, n, k, kind=kind, pow2=pow2)


@pytest.mark.parametrize("pow2", (False, True))
@pytest.mark.parametrize("layout", (X.MG_ROW_MAJOR, X.MG_COL_MAJOR))
@pytest.mark.parametrize("a_square", (False, True))
@pytest.mark.parametrize("b_square", (False, True))
def test_block_forms_whole_numbers(pow2, layout, a_square, b_square):
    """exact: every sum of whole numbers times powers of two fits FP32"""
    for m, n, k in ((1, 200, 300), (40, 150, 640), (150, 260, 400), (300, 520, 272)):
        check(m, n, k, layout, "f32", a_square, b_square, pow2, whole=True)


@pytest.mark.parametrize("ld,starts", (((304, 320), (0, 0, 0)), ((304, 320), (16, 32, 4)), ((301, 307), (0, 0, 0)), ((304, 304), (1, 0, 1)), ((304, 304), (0, 3, 3)),
                                       ((300, 300), (4, 8, 0))))
@pytest.mark.parametrize("pow2", (False, True))
def test_strides_and_alignment(ld, starts, pow2):
    for m, n in ((3, 130), (200, 300)):
        for kind in ("f32", "bf16"):
            check(m, n, 300, kind=kind, pow2=pow2, ld=ld, starts=starts, ldc=n + 5)
            check(m, n, 300, X.MG_COL_MAJOR, kind, True, False, pow2, ld=ld, starts=starts, ldc=m + 3)


@pytest.mark.parametrize("kind", ("f32", "f16", "bf16"))
@pytest.mark.parametrize("m,n,k", ((4, 70, 500), (140, 260, 512)))
def test_scalars(kind, m, n, k):
    for alpha, beta in ((1.0, 1.0), (0.5, -2.0), (-1.5, 0.0), (0.0, 0.5), (0.0, 0.0)):
        check(m, n, k, kind=kind, alpha=alpha, beta=beta)


@pytest.mark.parametrize("workspace", (False, True))
def test_long_sums(workspace):
    """few outputs and long sums: slices when there is a workspace; the last of them may be short or empty"""
    for m, n, k in ((1, 48, 40000), (20, 40, 33000), (130, 140, 20001), (128, 128, 16384), (256, 256, 9999)):
        for pow2 in (False, True):
            check(m, n, k, pow2=pow2, workspace=workspace)
    check(130, 140, 5000, kind="bf16", beta=1.0, workspace=workspace)


def test_no_sum():
    check(9, 20, 0, beta=0.5)
    check(9, 20, 0)


def test_larger():
    check(1100, 900, 1040, kind="bf16", pow2=True)
    check(1000, 1001, 999, X.MG_COL_MAJOR, "f16", False, False, True)
    check(520, 2050, 768, kind="f32", b_square=True)
    check(520, 2050, 768, kind="f32", b_square=False, pow2=False)


def test_nan_and_infinity_stay_in_their_rows():
    """a NaN element of A spoils its row of C, one of B its column, nothing else; an infinite scale likewise"""
    for m, n, k in ((20, 150, 300), (300, 290, 300)):
        rng = np.random.default_rng(2)
        a, A, SA = operand(rng, m, k, False, False, False, k, 0)
        b, B, SB = operand(rng, n, k, False, False, False, k, 0)
        A[3 * k + 299], B[130 * k + 5], SA[7, 1] = 0x7F, 0xFF, float("inf")
        c = torch.zeros(m, n, device="cuda")
        X.mg_block_gemm(X.MG_ROW_MAJOR, m, n, k, 1.0, X.MG_SCALES_ANY, X.MG_BLOCK_ROW, A, k, SA, SA.shape[1], X.MG_BLOCK_ROW, B, k, SB, SB.shape[1], 0.0, X.MG_F32, c, n)
        got = c.cpu().numpy()
        assert np.isnan(got[3]).all() and np.isnan(got[:, 130]).all() and not np.isfinite(got[7]).any()
        rest = np.delete(np.delete(got, [3, 7], 0), 130, 1)
        want, magnitudes = R.product(np.delete(a, [3, 7], 0), np.delete(b, 130, 0))
        assert (np.abs(rest - want) <= R.product_bound(want, magnitudes, k, "f32")).all()


def test_offsets_past_32_bits():
    """rows of A, of B and of C more than 2^32 bytes behind the first"""
    ld = (1 << 31) + 4096
    rng = np.random.default_rng(4)
    for m, n in ((3, 40), (40, 3)):
        k = 256
        q = {name: R.round_e4m3(rng.standard_normal((rows, k))) for name, rows in (("a", m), ("b", n))}
        s = {name: rng.uniform(0.5, 2, (rows, 2)).astype(np.float32) for name, rows in (("a", m), ("b", n))}
        far = "a" if m == 3 else "b"
        held = {}
        for name, rows in (("a", m), ("b", n)):
            lead = ld if name == far else k
            held[name] = torch.zeros((rows - 1) * lead + k, dtype=torch.uint8, device="cuda"), lead
            for r in range(rows):
                held[name][0][r * lead:r * lead + k] = torch.tensor(q[name][r]).cuda()
        ldc = (1 << 30) + 64 if m == 3 else n
        c = torch.zeros((m - 1) * ldc + n, device="cuda")
        X.mg_block_gemm(X.MG_ROW_MAJOR, m, n, k, 1.0, X.MG_SCALES_ANY, X.MG_BLOCK_ROW, held["a"][0], held["a"][1], torch.tensor(s["a"]).cuda(), 2,
                        X.MG_BLOCK_ROW, held["b"][0], held["b"][1], torch.tensor(s["b"]).cuda(), 2, 0.0, X.MG_F32, c, ldc)
        torch.cuda.synchronize()
        want, magnitudes = R.product(R.values(q["a"], s["a"], False), R.values(q["b"], s["b"], False))
        got = np.stack([c[r * ldc:r * ldc + n].cpu().numpy() for r in range(m)])
        assert (np.abs(got - want) <= R.product_bound(want, magnitudes, k, "f32")).all()
        del c, held
        torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------ experts

def experts_case(rng, counts, fan, extra):
    total, experts = sum(counts), len(counts)
    rows = -(-(total + extra) // fan) * fan
    source = np.full(rows, -1, np.int32)
    source[:total] = rng.permutation(rows)[:total]
    return np.cumsum([0] + counts).astype(np.int32), source, rows


COUNTS = ([3, 0, 1, 7], [0, 0, 0], [1], [130, 5, 0, 300], [128, 256], [16, 17, 15, 0, 33, 1], [2] * 70, [0] * 65 + [40])


@pytest.mark.parametrize("pow2", (False, True))
@pytest.mark.parametrize("kind", ("f32", "bf16"))
def test_grouped_rows(kind, pow2):
    for case, counts in enumerate(COUNTS):
        for n, k, fan, odd in ((200, 300, 2, 0), (130, 256, 1, 0), (64, 1040, 3, 0), (77, 129, 2, 3)):
            print(counts, n, k, fan, odd, flush=True)
            rng = np.random.default_rng(case)
            offsets, source, rows = experts_case(rng, counts, fan, 2)
            lead = -(-k // 16) * 16 + odd
            experts, total = len(counts), offsets[-1]
            a, A, SA = operand(rng, rows // fan, k, False, pow2, False, lead, 0)
            parts = [operand(rng, n, k, True, pow2, False, lead, 0) for _ in range(experts)]
            B, SB = torch.stack([p[1] for p in parts]), torch.stack([p[2] for p in parts])
            old = torch.tensor(rng.standard_normal((rows, n + 1))).to(TYPE[kind]).cuda()
            for beta, indexed in ((0.0, True), (0.5, fan > 1)):
                if not indexed and rows // fan < total:
                    continue
                c = old.clone()
                need = X.mg_block_gemm_grouped_workspace_bytes(experts, rows, n, k)
                ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
                X.mg_block_gemm_grouped(experts, torch.tensor(offsets).cuda(), rows, n, k, 1.5, kind_of_scales(pow2, kind), A, lead, SA, SA.shape[1],
                                        torch.tensor(source).cuda() if indexed else None, fan, X.MG_BLOCK_SQUARE, B, lead, B.shape[1], SB, SB.shape[2],
                                        SB.shape[1] * SB.shape[2], beta, CODE[kind], c, n + 1, ws)
                torch.cuda.synchronize()
                got = c.double().cpu().numpy()
                assert np.array_equal(got[total:], old.double().cpu().numpy()[total:]) and np.array_equal(got[:, n], old.double().cpu().numpy()[:, n])
                for e in range(experts):
                    lo, hi = offsets[e], offsets[e + 1]
                    index = source[lo:hi] // fan if indexed else np.arange(lo, hi)
                    want, magnitudes = R.product(a[index], parts[e][0], 1.5, beta, old[lo:hi, :n].double().cpu().numpy())
                    assert (np.abs(got[lo:hi, :n] - want) <= R.product_bound(want, magnitudes, k, kind)).all(), e


@pytest.mark.parametrize("pow2", (False, True))
@pytest.mark.parametrize("kind", ("f32", "bf16"))
def test_grouped_sums(kind, pow2):
    for case, counts in enumerate((*COUNTS, [1000, 1, 2000])):
        for m, n in ((130, 200), (16, 300), (1, 1), (260, 129)):
            print(counts, m, n, flush=True)
            rng = np.random.default_rng(case)
            experts, total = len(counts), sum(counts)
            rows, offsets = total + 3, np.cumsum([0] + counts).astype(np.int32)
            columns = X.mg_grouped_columns(rows, experts)
            stored, scales = {}, {}
            values = {}
            for name, high in (("a", m), ("b", n)):
                q = np.full((high, columns), 0x7F, np.uint8)
                s = np.full((high, columns // 128), np.nan, np.float32)
                for e in range(experts):
                    lo, count = int(offsets[e]), counts[e]
                    if count == 0:
                        continue
                    at, wide = R.group_column(lo, e), -(-count // 128) * 128
                    q[:, at:at + wide] = 0
                    q[:, at:at + count] = R.round_e4m3(rng.standard_normal((high, count)))
                    here = np.exp2(rng.integers(-6, 3, (high, wide // 128)).astype(np.float64))
                    s[:, at // 128:(at + wide) // 128] = here if pow2 else here * rng.uniform(1, 2, here.shape)
                    values[name, e] = R.values(q[:, at:at + count], s[:, at // 128:(at + wide) // 128], False)
                stored[name], scales[name] = torch.tensor(q).cuda(), torch.tensor(s).cuda()
            old = torch.tensor(rng.standard_normal((experts, m, n + 2))).to(TYPE[kind]).cuda()
            for beta in (0.0, 1.0):
                c = old.clone()
                need = X.mg_block_gemm_grouped_sum_workspace_bytes(experts, rows, m, n)
                ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
                X.mg_block_gemm_grouped_sum(experts, torch.tensor(offsets).cuda(), rows, m, n, 0.5, kind_of_scales(pow2, kind), stored["a"], columns,
                                            scales["a"], columns // 128, stored["b"], columns, scales["b"], columns // 128, beta, CODE[kind], c, n + 2, m * (n + 2), ws)
                torch.cuda.synchronize()
                got = c.double().cpu().numpy()
                assert np.array_equal(got[:, :, n:], old.double().cpu().numpy()[:, :, n:])
                for e in range(experts):
                    given = old[e, :, :n].double().cpu().numpy()
                    if counts[e] == 0:
                        assert np.array_equal(got[e, :, :n], given * beta)
                        continue
                    want, magnitudes = R.product(values["a", e], values["b", e], 0.5, beta, given)
                    assert (np.abs(got[e, :, :n] - want) <= R.product_bound(want, magnitudes, counts[e], kind)).all(), e


def test_no_rows_at_all():
    """a sum over nothing leaves beta * C; products of no rows leave C"""
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    c = torch.ones(2, 5, 6, device="cuda")
    X.mg_block_gemm_grouped_sum(2, offsets, 0, 5, 6, 1.0, X.MG_SCALES_ANY, None, 256, None, 2, None, 256, None, 2, 0.5, X.MG_F32, c, 6, 30)
    torch.cuda.synchronize()
    assert (c == 0.5).all()


def test_graph_replays():
    """captured once, replayed with eager work in between: the same numbers every time, also where slices are added"""
    for m, n, k in ((4, 256, 512), (130, 140, 20000)):
        rng = np.random.default_rng(6)
        _, A, SA = operand(rng, m, k, False, True, False, k, 0)
        _, B, SB = operand(rng, n, k, True, True, False, k, 0)
        c = torch.zeros(m, n, device="cuda")
        need = X.mg_block_gemm_workspace_bytes(m, n, k)
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        call = lambda: X.mg_block_gemm(X.MG_ROW_MAJOR, m, n, k, 1.0, X.MG_SCALES_POW2, X.MG_BLOCK_ROW, A, k, SA, SA.shape[1], X.MG_BLOCK_SQUARE, B, k, SB,  # noqa: E731
                                       SB.shape[1], 0.0, X.MG_F32, c, n, ws)
        call()
        torch.cuda.synchronize()
        want = c.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(3):
            c.zero_()
            ws.random_(0, 255)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(c, want)
