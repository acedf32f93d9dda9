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
