"""What the compiler gave the paged attention's kernels, read from the built library's kernel descriptions."""
import re
import subprocess

from test_encode_resources import READELF, code_objects, lib_path  # noqa: F401


def instances(path, tmp_path):
    """(head size, subspaces, query heads, e4m3, wavefronts) of attend_pages_kernel -> registers, spilled registers."""
    out = {}
    for n, blob in enumerate(code_objects(path)):
        if b"attend_pages_kernel" not in blob:
            continue
        file = tmp_path / f"{n}.co"
        file.write_bytes(blob)
        text = subprocess.run([READELF, "--notes", str(file)], check=True, stdout=subprocess.PIPE, text=True).stdout
        for part in text.split(".agpr_count:")[1:]:
            name = re.search(r"\.name:\s+\S*attend_pages_kernelILi(\d+)ELi(\d+)ELi(\d+)ELb(\d)ELi(\d)E", part)
            if name:
                value = lambda key: int(re.search(rf"\.{key}:\s+(\d+)", part).group(1))
                out[tuple(int(x) for x in name.groups())] = value("vgpr_count"), value("vgpr_spill_count")
    return out


def test_registers_of_the_paged_attention(lib_path, tmp_path):  # noqa: F811
    """128 registers: two workgroups of eight wavefronts to a compute unit.  80 at d_k = 64 for one or two query heads with at most 16 tables
    between them: three workgroups.  Any number where 128 KB of tables leave room for one.  Few registers are spilled, and only by two heads
    at d_k = 64, m = 8 and d_k = 128, m = 16."""
    found = instances(lib_path, tmp_path)
    assert len(found) >= 2 * 4 * 4 * 2
    for (d_k, m, G, _, _), (registers, spilled) in found.items():
        most = 256 if G * m >= 128 else 80 if d_k == 64 and G <= 2 and G * m <= 16 else 128
        may_spill = 6 if (d_k, m, G) == (64, 8, 2) else 4 if (d_k, m, G) == (128, 16, 2) else 0
        assert registers <= most and spilled <= may_spill, (d_k, m, G, registers, spilled)
