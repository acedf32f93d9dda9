"""Registers of the operators' kernels (no GPU): what their launches count on."""
import re

from test_device_assembly import assembly  # noqa: F401  (the library's device code)


def kernels(lines):
    """name -> vgpr_count, vgpr_spill_count, private_segment_fixed_size of every kernel."""
    out, entry = {}, {}
    for line in lines:
        m = re.match(r"\s+(- )?\.(\w+):\s+(\S+)", line)
        if not m:
            continue
        if m.group(2) == "agpr_count":
            entry = {}
        entry[m.group(2)] = m.group(3)
        if m.group(2) == "wavefront_size":
            out[entry["name"]] = {k: int(entry[k]) for k in ("vgpr_count", "vgpr_spill_count", "private_segment_fixed_size")}
    return out


def test_registers_of_the_operators(assembly):  # noqa: F811
    """Distillation: a row in registers, beside what settles it, without scratch, and as many workgroups on a compute unit as
    the launch is made for.  Verification without scratch.  Scans: at most 8 registers in scratch (fp32 sigmoid in chains, 16-bit
    sigmoid gradients of one tile)."""
    k = kernels(assembly)
    distill = {n: v for n, v in k.items() if "distill_rows_kernel" in n}
    assert len(distill) == 18
    for name, v in distill.items():
        threads, held = (int(x) for x in re.search(r"Lj(\d+)ELj(\d+)E", name).groups())
        waves = 8 if held == 4 else 6 if (threads, held) == (512, 8) else 4       # of a SIMD's 512 registers
        assert v["vgpr_spill_count"] == v["private_segment_fixed_size"] == 0 and v["vgpr_count"] <= 512 // waves // 8 * 8, (name, v)
    verify = {n: v for n, v in k.items() if "verify_kernel" in n}
    assert len(verify) == 3 and all(v["private_segment_fixed_size"] == 0 and v["vgpr_count"] <= 128 for v in verify.values()), verify
    scan = {n: v for n, v in k.items() if "scan_tile" in n or "scan_channel" in n}
    assert len(scan) == 36 and all(v["vgpr_spill_count"] <= 8 for v in scan.values()), scan


def test_registers_of_the_learning_steps_operators(assembly):  # noqa: F811
    """Gated delta rule: registers in scratch only where the kernels' comments say so, and as many workgroups on a compute unit as the
    launches are made for.  Embedding and clipping without scratch, eight waves of a SIMD (slices of 16 bits seven, the sort by one
    workgroup four)."""
    k = kernels(assembly)

    def of(name):
        return {n: v for n, v in k.items() if re.search(r"\d" + name, n)}

    def held(n):    # registers in scratch at most, of the pieces and of the gradient's last kernel
        size, name = 4 if "kernelIf" in n else 2, "gradients" if "gradients" in n else "pieces"
        if name == "pieces":
            return 8 if size == 4 and "Lj4ELj" in n and "back" not in n else 0
        width, waves, whole = re.search(r"Lj(\d)ELj(\d)ELb(\d)", n).groups()
        if (width, waves) == ("2", "8"):
            return 0
        narrow = width == "2"
        if size == 4:
            return (16 if narrow else 40) if whole == "1" else (52 if narrow else 72)
        return (0 if narrow else 6) if whole == "1" else (8 if narrow else 28)

    pieces, gradients, prepare = of("delta_pieces_(?:back_)?kernel"), of("delta_gradients_kernel"), of("delta_prepare_kernel")
    assert (len(pieces), len(gradients), len(prepare)) == (18, 18, 13)
    for n, v in {**pieces, **gradients}.items():
        assert v["vgpr_spill_count"] <= held(n), (n, v, held(n))
        # (one wave a SIMD of the pieces, two of the gradient)
        assert v["vgpr_count"] <= (512 if n in pieces else 256), (n, v)
    for n, v in prepare.items():
        workgroups = 2 if "kernelIfLj4" in n else 3
        assert v["vgpr_spill_count"] == v["private_segment_fixed_size"] == 0 and v["vgpr_count"] <= 512 // workgroups // 8 * 8, (n, v)
    rest = {n: v for name in ("delta_steps_kernel", "embed_kernel", "embed_slices2?_kernel", "embed_rows_kernel", "sort_\\w+_kernel",
                              "clip_norm_kernel", "clip_scale_kernel") for n, v in of(name).items()}
    assert len(rest) == 19, sorted(rest)
    for n, v in rest.items():
        waves = 4 if "delta_steps" in n or "sort_alone" in n else 7 if "slices_" in n else 8
        assert v["vgpr_spill_count"] == v["private_segment_fixed_size"] == 0 and v["vgpr_count"] <= 512 // waves // 8 * 8, (n, v)
