"""Which tiles and cuts the calls of the operators around the network take, and that the sizes of the GPU tests take all of them (no GPU needed)."""
from paper_2112_05387_amd import binding as B
from tests.test_gpu_operator_tiles import CLASSES, MATRICES


def _plans(dtype):
    for n, c, v in CLASSES[dtype]:
        d = B.lp_linear_ce_desc(n, c, v, B.LP_BF16 if dtype == "bf16" else B.LP_F32, 0, 0, 0)
        yield (n, c, v), B.lp_debug_linear_ce_plan(d, False), B.lp_debug_linear_ce_plan(d, True)


def _taken(dtype):
    taken = {}
    for shape, forward, (direct, cut, pieces, tile, _, tx, sx, tw, sw) in _plans(dtype):
        assert direct == 0, shape
        for key in (("loss", forward[1], forward[3]), ("probabilities", cut, tile, pieces > 1), ("dfeatures", tx, sx > 1, pieces > 1), ("dweight", tw, sw > 1, pieces > 1)):
            taken.setdefault(key, shape)
    return taken


def test_classifier_tiles_bf16():
    taken = _taken("bf16")
    want = [("loss", 0, t) for t in range(4)] + [("loss", 1, t) for t in (2, 3)]
    want += [("probabilities", 0, t, many) for t in range(4) for many in (False, True)] + [("probabilities", 1, t, False) for t in (2, 3)]
    want += [("dfeatures", t, cut, many) for t in range(3) for cut in (False, True) for many in (False, True)]
    want += [("dfeatures", 3, False, False), ("dfeatures", 3, True, False), ("dfeatures", 3, True, True)]
    want += [("dweight", t, cut, many) for t in range(3) for cut in (False, True) for many in (False, True)]
    assert set(want) == set(taken), (set(want) - set(taken), set(taken) - set(want))


def test_classifier_tiles_f32():
    taken = _taken("f32")
    want = [("loss", 0, 4), ("loss", 0, 5), ("loss", 1, 5), ("probabilities", 1, 5, False)]
    want += [("probabilities", 0, t, many) for t in (4, 5) for many in (False, True)]
    want += [(name, t, cut, many) for name in ("dfeatures", "dweight") for t in (4, 5) for cut in (False, True) for many in (False, True)]
    assert set(want) == set(taken), (set(want) - set(taken), set(taken) - set(want))


def test_reduction_of_the_weights_over_many_tiles():
    """256 x 256 tiles of dweight over more k-tiles than are loaded ahead, the last one ragged, words of the row mask behind each other."""
    plan = dict((s, b) for s, _, b in _plans("bf16"))[(1000, 2040, 50000)]
    assert plan[7:9] == [0, 1] and 1000 % 64 and 1000 // 64 > 4


def test_orthogonalisation_tiles():
    plans = {}
    for shapes in MATRICES:
        mats = (B.lp_matrix * len(shapes))(*[B.lp_matrix(r, c, B.LP_F32, B.LP_F32, 0x10000000, 0x10000000, 0, 0) for r, c in shapes])
        square, step, small = B.lp_debug_orthogonalize_plan(mats)
        assert small == 0
        plans.setdefault((step, shapes[0][0] > shapes[0][1]), shapes)
        plans.setdefault(("symmetric", square), shapes)
    assert set(plans) == {(t, tall) for t in range(4) for tall in (False, True)} | {("symmetric", t) for t in (0, 2, 3)}, plans


def test_workspace_of_a_gradient_that_needs_no_sums():
    """dfeatures comes whole out of its product: no partial results of it are held.  What is: three parts of the probabilities, sums of the other classes (a float
    for 128 classes of a row) and over the rows (one for 64 rows of a class), the row mask, a float a row, and alignment."""
    for n, c, v in ((20000, 1024, 4096), (8000, 2048, 20000), (2048, 2048, 8192)):
        d = B.lp_linear_ce_desc(n, c, v, B.LP_BF16, 0, 0, 0)
        plan = B.lp_debug_linear_ce_plan(d, True)
        assert plan[2] == 1 and plan[6] == 1 and plan[8] == 1
        wide = v + 256
        assert B.lp_linear_ce_workspace_bytes(d, True) <= 6 * n * wide + 4 * n * (wide // 128 + 2) + 4 * (n // 64 + 4) * wide + 5 * n + 8192 < 6 * n * v + 4 * n * c
