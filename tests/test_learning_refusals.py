"""What the learning step's operators refuse before anything is launched (no GPU)."""
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
