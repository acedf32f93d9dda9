"""Which launches the operators make, on a HIP runtime that only records them (no GPU)."""
import recorded_hip

SCAN = """
def scan(S, T, D, back=False, workspace=True, dtype=1, gate=1):
    a = [S, T, D, dtype, gate, memory(), T * D, D, memory(), T * D, D, None, None]
    if back:
        a += [memory(), memory(), None, memory(), T * D, D, memory(), T * D, D, None]
    else:
        a += [None, memory(), None, None]
    rc = call("apex_gated_scan_backward" if back else "apex_gated_scan", *a, memory() if workspace else None, None)
    return rc, launches()

def bytes_of(entry, *sizes):
    n = C.c_size_t(0)
    assert call(entry, *sizes, C.byref(n)) == 0
    return n.value
"""


def test_scan_by_channel_by_tile_and_by_chains_of_tiles(tmp_path):
    out = recorded_hip.run(tmp_path, SCAN + """
result = [[scan(S, T, D, back)[1] for S, T, D in ((64, 1, 1000), (3, 11, 64), (3, 12, 130), (64, 96, 1024), (5, 128, 100),
                                                  (2, 129, 300), (4, 8192, 2048))] for back in (False, True)]
""")
    for back, name in ((0, "scan_"), (1, "scan_")):
        for l in out[back]:
            assert len(l) == 1 and ("back" in l[0]["kernel"]) == bool(back)
        kinds = ["channel" if "scan_channel" in l[0]["kernel"] else "tile" for l in out[back]]
        assert kinds == ["channel", "channel", "tile", "tile", "tile", "tile", "tile"]
        shape = [(l[0]["grid"], l[0]["block"]) for l in out[back]]
        assert shape[:2] == [(64 * 16, 64), (3, 64)]                     # a thread per channel
        assert shape[2:5] == [(3 * 2, 128), (64 * 8, 768), (5, 1024)]    # a workgroup per 128 channels
        assert shape[5:] == [(2 * 3 * 3, 512), (4 * 16 * 128, 512)]      # ... and 64 steps


def test_scan_workspace_where_tiles_are_chained(tmp_path):
    out = recorded_hip.run(tmp_path, SCAN + """
need = lambda S, T, D: bytes_of("apex_gated_scan_workspace_bytes", S, T, D)
result = [need(9, 128, 5000), need(1, 129, 1), need(2, 129, 1), need(2, 300, 200), need(2, 300, 4096)] + [
    scan(2, 129, 8, back, workspace=False)[0] for back in (0, 1)] + [scan(2, 128, 8, back, workspace=False)[0] for back in (0, 1)]
""")
    assert out[0] == 0 and 0 < out[1] < out[2] < out[3] < out[4]
    head = out[1] - 3 * 3 * 128 * 8
    assert out[3] == head + 2 * 5 * 256 * 3 * 8 and out[4] == head + 2 * 5 * 4096 * 3 * 8
    assert out[5:] == [-1, -1, 0, 0]


def test_distillation_holds_a_row_in_as_few_threads_as_it_can(tmp_path):
    out = recorded_hip.run(tmp_path, """
def distill(N, V, dtype=1):
    assert call("apex_distill_topk", N, V, 8, dtype, memory(), V, memory(), 0, memory(), None, None, 1.0, memory(), None, memory(), V,
                None, None) == 0
    return launches()
result = [distill(*a) for a in ((5, 1), (5, 8199), (3000, 8200), (3000, 32775), (3000, 32776), (3000, 65543), (3000, 65544),
                                (3000, 131079), (3000, 131080), (3000, 1 << 20), (200, 32775), (200, 65544), (3000, 16388, 0))]
""")
    assert [l[0]["block"] for l in out] == [256, 256, 512, 512, 512, 512, 1024, 1024, 1024, 1024, 1024, 1024, 512]
    assert all(len(l) == 1 for l in out)
    held = [int(l[0]["kernel"].split("Lj")[2].split("E")[0]) for l in out]
    assert held == [4, 4, 8, 8, 16, 16, 16, 16, 16, 16, 8, 16, 16]
    assert ["Lb1" in l[0]["kernel"] for l in out] == [i in (8, 9) for i in range(13)]      # rows of which a part is read twice
    assert [l[0]["grid"] for l in out[:3]] == [5, 5, 3000]


def test_verification_shares_rows_among_workgroups(tmp_path):
    out = recorded_hip.run(tmp_path, """
def verify(B, V):
    assert call("apex_verify_draft", B, 2, V, 0, memory(), 3 * V, V, memory(), 2 * V, V, memory(), memory(), None, memory(), memory(),
                memory(), None) == 0
    return launches()[0]["grid"]
result = [verify(*a) for a in ((1, 1), (1, 4096), (1, 4097), (1, 131072), (1, 1 << 20), (64, 32768), (256, 128001), (5000, 100000),
                               (5000, 1 << 20))]
""")
    assert out == [1, 1, 2, 32, 64, 64 * 8, 256 * 16, 5000, 5000 * 2]
