"""In which order the launches of clipping go through the tensors: what a launch's argument says, on a HIP runtime that only records (no
GPU)."""
import recorded_hip

# A clipping kernel's argument, by words of 32 bits: tensors, pieces, before, all, piece, max_norm, flags, (pad), norm, space, and from
# word 12 on eight words a tensor: gradient, output, elements, first piece, type.
WORDS = r"""
  if (strstr(name, "clip_")) {
    const uint32_t *w = (const uint32_t *)args[0];
    for (uint32_t i = 0; i < w[0]; ++i) {
      const uint32_t *t = w + 12 + 8 * i;
      line("tensor %u %u %u %lu %u\n", w[1], w[2], w[4], (unsigned long)(t[4] | (unsigned long)t[5] << 32), t[6]);
    }
  }
"""

CLIP = """
def clip(sizes):
    n = len(sizes)
    array = lambda t, x: (t * n)(*x)
    assert call("apex_clip_gradients", n, array(C.c_void_p, [memory() for _ in sizes]), array(C.c_void_p, [memory() for _ in sizes]),
                array(C.c_uint64, sizes), array(C.c_int, [0] * n), 1.0, memory(), memory(), None) == 0
    out = []
    for c in take():
        if c[0] == "launch":
            out.append(("norm" if "norm" in c[5] else "scale", []))
        elif c[0] == "tensor":
            pending.append(c[1:])
            continue
        out[-1][1].extend(pending)
        pending.clear()
    return out
pending = []
"""


def places(launch):
    """(elements of the tensor, piece of it) by workgroup: workgroup b of the norm takes piece b of the table, of the scaling the b-th
    from its end."""
    kind, table = launch
    pieces = table[0][0]
    out = []
    for b in range(pieces):
        at = b if kind == "norm" else pieces - 1 - b
        i = max(i for i, t in enumerate(table) if t[4] <= at)
        out.append((table[i][3], at - table[i][4]))
    return out


def test_the_scaling_goes_backwards_through_what_the_norm_went_through(tmp_path, monkeypatch):
    launch = '  line("launch %lu %u %u %u %.200s\\n", (unsigned long)st, g.x, g.y, b.x, name);\n'
    assert recorded_hip.SOURCE.count(launch) == 1
    monkeypatch.setattr(recorded_hip, "SOURCE", recorded_hip.SOURCE.replace(launch, WORDS + launch))
    # (every tensor has a size of its own; some have none, some several pieces)
    sizes = [[10, 4, 3], [20000], [9000, 0, 30000, 1, 8192, 8193], [0, 0, 5], list(range(1, 250)), [70000] + [0] * 100 + list(range(1, 98))]
    out = recorded_hip.run(tmp_path, CLIP + "result = [clip(s) for s in %r]\n" % sizes)
    for s, launches in zip(sizes, out):
        norm, scale = ([p for l in launches if l[0] == kind for p in places(l)] for kind in ("norm", "scale"))
        assert norm == [(n, p) for n in s for p in range(-(-n // 8192))], s
        assert scale == norm[::-1], s
