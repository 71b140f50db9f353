"""The choice of the kernel for a product of 16-bit matrices, on the host: every kernel is taken somewhere in the GPU tests, slices fit their room and cover the sum."""
import random

from tests.linear_choice import choices, together


def padded(v):
    return -(-v // 64) * 64


def block(tokens, width, hidden):
    both = 2 * padded(hidden)
    return [("kk", "gated", tokens, -(-hidden // 16) * 32, width), ("kk", "store", tokens, width, hidden), ("kn", "gated_grad", tokens, hidden, width), ("kn", "store", tokens, width, both),
            ("nn", "store", both, width, tokens), ("nn", "store", width, hidden, tokens)]


def loss(tokens, width, vocab):
    return [("kk", "scores", tokens, vocab, width), ("kk", "scores_grad", tokens, vocab, width), ("kn", "store", tokens, width, vocab), ("nn", "store", vocab, width, tokens)]


def ends(products):
    """the products of a call that go together where that pays: (rows, cols, k) of the one with its operand across the sum, and of those with both"""
    sizes = [p[2:] for p in products if p[:2] == ("kn", "store")] + [p[2:] for p in products if p[0] == "nn"]
    return (*(sizes + [(0, 0, 0)])[:3], 1 << 40)


def test_the_gpu_tests_reach_every_kernel():
    """gradients wanted one by one too, whose products are not asked to go together"""
    from tests import test_gpu_layers as G
    calls = [block(*c) for c in G.BLOCKS + G.LARGE_BLOCKS] + [loss(*c) for c in G.LOSSES + G.LARGE_LOSSES]
    joined = together([ends(c) for c in calls])
    assert {(j[0], j[1] > 1) for j in joined} == {("any", False), ("128", False), ("128", True), ("64", False), ("64", True)}
    asked = [p for c, j in zip(calls, joined) for p in c if j[0] == "any" or p[0] == "kk" or p[1] != "store"]
    asked += [p for c in G.ONE_GRADIENT for p in block(*c)]
    taken = {(form, end, kernel) for (form, end, *_), (kernel, _, _) in zip(asked, choices(asked))}
    # what a block keeps passes the caches by from 128 MB on, on the largest tiles
    tokens, width, hidden = G.LARGE_BLOCKS[-1]
    assert tokens // 16 * (hidden // 16) * 1152 >= 1 << 27 and [c[0] for c in choices([block(tokens, width, hidden)[i] for i in (0, 2)])] == ["256", "256"]
    pairs = {(form, end) for form, end, *_ in asked}
    missing = {(*pair, tile) for pair in pairs for tile in ("256", "128", "64", "64 twice")} - taken
    assert not missing, missing
    assert sum(t[2] == "128 deep" for t in taken) >= 3, taken
    assert {("kk", end, "few") for end in ("store", "gated", "scores")} <= taken


def test_both_matrices_of_a_sum_are_read_on_every_tile():
    """by the GPU test whose gate and up weights lie at different distances"""
    got = choices([block(*c)[3] for c in ((1000, 1000, 2000), (2100, 4000, 520), (4000, 1500, 700), (1500, 2000, 1000))])
    assert [g[0] for g in got] == ["64 twice", "256", "128", "128 deep"]


def test_products_that_go_together():
    """both sides were measured (csrc/linear_plan.h); slices cover the sum and fit their room"""
    got = together([((333, 1001, 4096), (4096, 1001, 333), (1001, 1999, 333), 1 << 30), ((64, 512, 2048), (2048, 512, 64), (512, 1024, 64), 1 << 30),
                    ((1024, 1024, 4096), (4096, 1024, 1024), (1024, 2048, 1024), 1 << 30), ((4096, 1024, 4096), (4096, 1024, 4096), (1024, 2048, 4096), 1 << 30),
                    ((333, 1001, 4096), (0, 0, 0), (0, 0, 0), 1 << 30), ((8192, 2048, 16384), (16384, 2048, 8192), (2048, 8192, 8192), 1 << 40)])
    assert [g[0] for g in got] == ["128", "64", "128", "any", "any", "any"] and [g[1] for g in got[:3]] == [4, 8, 2]
    rng = random.Random(2)
    size = lambda most: int(round(most ** rng.random()))  # noqa: E731
    asked = [(tuple(size(9000) for _ in range(3)), (size(20000), size(3000), size(3000)), (0, 0, 0), rng.choice((0, 1 << 16, 1 << 20, 1 << 30))) for _ in range(1000)]
    taken = 0
    for (first, _, _, room), (kernel, slices, each) in zip(asked, together(asked)):
        if kernel == "any":
            continue
        taken += slices > 1
        assert each % 64 == 0 and (slices - 1) * each < first[2] <= slices * each and (slices == 1 or slices * first[0] * padded(first[1]) * 4 <= room)
    assert taken > 20


def test_slices_cover_the_sum_and_fit_their_room():
    rng = random.Random(1)
    asked = []
    for _ in range(3000):
        size = lambda most: int(round(most ** rng.random()))  # noqa: E731
        form = rng.choice(("kk", "kn", "nn"))
        end = rng.choice({"kk": ("store", "gated", "scores", "scores_grad"), "kn": ("store", "gated_grad"), "nn": ("store",)}[form])
        asked.append((form, end, size(20000), size(70000), size(70000), rng.random() < 0.7, rng.choice((0, 1 << 20, 1 << 24, 1 << 28, 1 << 40))))
    split = 0
    for (form, end, rows, cols, k, aligned, room), (kernel, slices, each) in zip(asked, choices(asked)):
        assert each % 64 == 0 and (slices - 1) * each < k <= slices * each
        assert aligned == (kernel not in ("any", "any few"))
        assert slices == 1 or (end == "store" and slices * rows * padded(cols) * 4 <= room)
        assert kernel not in ("few", "any few") or (form == "kk" and rows <= 32)
        split += slices > 1
    assert split > 100


def test_measured_choices():
    """both sides were measured: 2048^3 30.2 us on 128, 21.7 on 128 deep; 4096 x 4096 x 2048 76 and 57 on 256; 8192 x 1024 x 1024 28 on 256, 21.5 on 128; 512 x 2048 x 2048
    20 on 128 deep, 10.7 on 64, 9.3 with two sets of wavefronts; 256 x 256 x 8192 39 in one slice of 64, 13 in eight and more"""
    got = choices([("kk", "store", 2048, 2048, 2048), ("kk", "store", 4096, 4096, 2048), ("kk", "store", 8192, 1024, 1024), ("kk", "store", 512, 2048, 2048), ("nn", "store", 256, 256, 8192)])
    assert [g[0] for g in got] == ["128 deep", "256", "128", "64 twice", "64"] and got[4][1] >= 8 and [g[1] for g in got[:4]] == [1] * 4
