"""Which launches the learning step's operators make, on a HIP runtime that only records them (no GPU)."""
import recorded_hip

DELTA = """
def delta(S, T, Hk, H, Dk, Dv, back=False, dtype=1, workspace=True):
    a = [S, T, Hk, H, Dk, Dv, dtype]
    for n in (Hk * Dk, Hk * Dk, H * Dv):
        a += [memory(), T * n, n]
    a += [memory(), memory(), 1.0, None, None]
    if back:
        a += [memory(), memory(), None]
        for n in (Hk * Dk, Hk * Dk, H * Dv):
            a += [memory(), T * n, n]
        a += [memory(), memory(), None]
    else:
        a += [None, memory(), None, None]
    rc = call("apex_delta_rule_backward" if back else "apex_delta_rule", *a, memory() if workspace else None, None)
    return rc, [(l["kernel"], l["grid"], l["block"]) for l in launches()]
"""


def test_delta_rule_by_steps_and_by_pieces(tmp_path):
    out = recorded_hip.run(tmp_path, DELTA + """
result = [delta(64, 1, 16, 16, 128, 128), delta(2, 8, 1, 3, 16, 65, workspace=False), delta(2, 9, 1, 3, 16, 65), delta(2, 17, 1, 3, 16, 65, workspace=False),
          delta(4, 8192, 8, 16, 128, 128), delta(4, 8192, 8, 16, 128, 128, back=True),
          delta(64, 16, 8, 8, 64, 64), delta(64, 17, 8, 8, 64, 64), delta(32, 16, 8, 8, 64, 64), delta(33, 16, 8, 8, 64, 64)]
""")
    assert [r for r, _ in out] == [0, 0, 0, -1, 0, 0, 0, 0, 0, 0]
    names = [[k for k, _, _ in l] for _, l in out]
    assert ["steps" in n[0] for n in names[:2]] == [True, True] and [len(n) for n in names] == [1, 1, 2, 0, 2, 3, 1, 2, 2, 1]
    assert out[0][1][0][1:] == [64 * 16 * 2, 256] and out[1][1][0][1:] == [2 * 3 * 2, 256]
    for l in (out[2][1], out[4][1], out[5][1]):
        assert "prepare" in l[0][0] and "pieces" in l[1][0]
    # a workgroup per head and 16 or 32 columns, eight heads at a time
    assert out[2][1][1][1:] == [8 * 5, 128] and out[4][1][1][1:] == out[5][1][1][1:] == [64 * 4, 256]
    assert out[4][1][0][1] == 4 * 128 * 16 and "gradients" in out[5][1][2][0] and out[5][1][2][1] == 4 * 128 * 8


def test_embedding_gradient_sorts_alone_or_by_tiles(tmp_path):
    out = recorded_hip.run(tmp_path, """
def back(N, V, D=64):
    assert call("apex_embedding_backward", N, V, D, 0, memory(), D, memory(), 1.0, 0, memory(), D, memory(), None) == 0
    return [(l["kernel"].split("kernel")[0][-12:], l["grid"]) for l in launches()]
result = [back(1, 1), back(8192, 50000), back(70, 2047), back(8192, 2048), back(8193, 2047), back(8193, 2048), back(65536, 5)]
""")
    kinds = [[next(w for w in ("alone", "count", "tiles", "place", "slices2", "slices", "rows") if w in k) for k, _ in l] for l in out]
    assert kinds[0] == kinds[1] == kinds[2] == kinds[3] == ["alone", "slices", "rows"]
    passes = ["count", "tiles", "place"]
    assert kinds[4] == passes + ["slices", "rows"] and kinds[5] == passes * 2 + ["slices", "rows"]
    assert kinds[6] == passes + ["slices", "slices2", "rows"]


def test_clipping_in_launches_of_many_tensors(tmp_path):
    out = recorded_hip.run(tmp_path, """
def clip(sizes, max_norm=1.0, out=True):
    n = len(sizes)
    array = lambda t, x: (t * max(n, 1))(*x)
    p = [memory() for _ in sizes]
    assert call("apex_clip_gradients", n, array(C.c_void_p, p), array(C.c_void_p, [memory() for _ in sizes] if out else p), array(C.c_uint64, sizes),
                array(C.c_int, [0] * n), max_norm, memory(), memory(), None) == 0
    return [("norm" if "norm" in l["kernel"] else "scale", l["grid"]) for l in launches()]
result = [clip([]), clip([0, 0]), clip([1]), clip([8192, 8193]), clip([10] * 200), clip([10] * 3, float("inf"), out=False), clip([10] * 3, float("inf")),
          clip([1 << 30] * 2)]
""")
    assert out[0] == out[1] == [["norm", 1]] and out[2] == [["norm", 1], ["scale", 1]] and out[3] == [["norm", 3], ["scale", 3]]
    assert out[4] == [["norm", 96], ["norm", 96], ["norm", 8], ["scale", 96], ["scale", 96], ["scale", 8]]
    assert out[5] == [["norm", 3]] and out[6] == [["norm", 3], ["scale", 3]]
    assert out[7][0][1] <= 4096 + 2 and out[7][0] == ["norm", out[7][1][1]]
