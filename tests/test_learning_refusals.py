"""What the learning step's operators refuse before anything is launched (no GPU)."""
import pytest
import torch

import recorded_hip

CLIP = """
def clip(parts, max_norm=1.0):
    "parts: (gradient's address, output's, elements)."
    n = len(parts)
    array = lambda t, x: (t * max(n, 1))(*x)
    rc = call("apex_clip_gradients", n, array(C.c_void_p, [p[0] for p in parts]), array(C.c_void_p, [p[1] for p in parts]),
              array(C.c_uint64, [p[2] for p in parts]), array(C.c_int, [0] * n), max_norm, memory(), memory(), None)
    return rc, len(launches())
a, b, c = memory(), memory(), memory()
"""


def test_clipping_over_tensors_that_are_written_twice(tmp_path):
    """In place or not: the same tensor named twice, one that lies within another, an output over another one's gradient."""
    out = recorded_hip.run(tmp_path, CLIP + """
inf = float("inf")
bad = [clip([(a, a, 100), (a, a, 100)]), clip([(b, b, 5), (a, a, 100), (a + 396, a + 396, 7)]), clip([(a + 40, a + 40, 3), (b, b, 9), (a, a, 100)]),
       clip([(a, c, 100), (b, c, 100)]), clip([(a, c, 100), (b, c + 396, 100)]), clip([(a, b, 100), (c, a + 396, 1)]), clip([(a, a + 4, 100)]),
       clip([(a, a, 100), (b, a + 40, 1)]), clip([(a, b, 10), (b, a, 10)], inf), clip([(a, a, 100), (b, c, 9), (c + 32, c + 400, 1)])]
good = [clip([(a, a, 100), (b, b, 100)]), clip([(a + 400, a + 400, 7), (a, a, 100)]), clip([(a, c, 100), (a, c + 400, 100)]), clip([(a, b, 100), (a + 40, c, 3)]),
        clip([(a, a, 100), (a, a, 100)], inf), clip([(a, a, 0), (a, a, 0), (a, a, 4)]), clip([(a, a + 400, 100)]), clip([])]
result = bad, good
""")
    assert out[0] == [[-1, 0]] * 10
    assert [rc for rc, _ in out[1]] == [0] * 8 and [n for _, n in out[1]] == [2, 2, 2, 2, 1, 2, 2, 1]


@pytest.fixture(scope="module")
def apex():
    from paper_1803_00933_amd import apex
    return apex


def clip_into(apex, grad, out):
    space = torch.zeros(1)
    apex.clip_gradients([grad], 1.0, out=[out], norm=space, workspace=space)


LAID_OUT = [((1, 8), (8, 1), (1, 1)), ((4, 1, 3), (3, 3, 1), (3, 50, 1)), ((5, 1), (1, 1), (1, 7)), ((1,), (1,), (9,)), ((0, 4), (4, 1), (1, 1))]


@pytest.mark.parametrize("sizes,strides,others", LAID_OUT, ids=str)
def test_clipping_into_tensors_of_the_same_layout(apex, sizes, strides, others):
    """A dimension of one element has any stride: these go on to the binding, which wants tensors of the GPU."""
    a, b = (torch.zeros(100).as_strided(sizes, s) for s in (strides, others))
    for x, y in ((a, b), (b, a)):
        with pytest.raises(AssertionError, match="dense tensors of a floating type"):
            clip_into(apex, x, y)


@pytest.mark.parametrize("grad,out", [((6,), (1, 6)), ((2, 6), (12,)), ((1, 6), (6, 1)), ((2, 3), (3, 2)), ((4,), (5,))], ids=str)
def test_clipping_into_tensors_of_other_sizes(apex, grad, out):
    with pytest.raises(ValueError, match="laid out"):
        clip_into(apex, torch.zeros(grad), torch.zeros(out))
    with pytest.raises(ValueError, match="laid out"):
        clip_into(apex, torch.zeros((3, 4)), torch.zeros((4, 3)).t())


def test_clipping_into_another_layout_of_one_stride(apex):
    """[6,1] and [1,6] in memory with the same strides: sizes count."""
    x = torch.zeros(50)
    with pytest.raises(ValueError, match="laid out"):
        clip_into(apex, x.as_strided((6, 1), (1, 1)), x.as_strided((1, 6), (1, 1)))
