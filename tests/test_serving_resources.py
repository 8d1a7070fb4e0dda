"""What the compiler gave the kernels of chunks, attention sums, eviction and beam selection, read from the built library's kernel descriptions."""
import re
import subprocess

import pytest

from test_encode_resources import READELF, code_objects, lib_path  # noqa: F401

KERNELS = ("chunk_kernel", "chunk_few_kernel", "weigh_kernel", "evict_pick_kernel", "evict_move_kernel", "select_rows_kernel", "select_merge_kernel")


@pytest.fixture(scope="module")
def instances(lib_path, tmp_path_factory):  # noqa: F811
    """(kernel, mangled template arguments) -> registers, spilled registers, threads of a workgroup."""
    out = {}
    for n, blob in enumerate(code_objects(lib_path)):
        if not any(k.encode() in blob for k in KERNELS):
            continue
        file = tmp_path_factory.mktemp("code") / f"{n}.co"
        file.write_bytes(blob)
        text = subprocess.run([READELF, "--notes", str(file)], check=True, stdout=subprocess.PIPE, text=True).stdout
        for part in text.split(".agpr_count:")[1:]:
            name = re.search(r"\.name:\s+_ZN6lookat\d+(\w+?_kernel)(I\S*?E|)E", part)
            if name and name.group(1) in KERNELS:
                value = lambda key: int(re.search(rf"\.{key}:\s+(\d+)", part).group(1))  # noqa: B023, E731
                out[name.group(1), name.group(2)] = value("vgpr_count"), value("vgpr_spill_count"), value("max_flat_workgroup_size")
    return out


def test_all_kernels_are_there(instances):
    assert {k for k, _ in instances} == set(KERNELS)


def test_registers(instances):
    """A workgroup's wavefronts fit their SIMDs' 512 registers; two wavefronts to a SIMD where a workgroup has no more than eight."""
    for key, (registers, _, threads) in instances.items():
        assert registers * max(1, threads // 256) <= 512, (key, registers, threads)
        if key[0].startswith("chunk"):
            assert registers <= 256, (key, registers)


def test_spilled_registers(instances):
    """None, but some by chunks at d_k = 128 (fp32 rows; 256 rows of e4m3) and by the choice of up to 32 tokens a thread."""
    for (kernel, args), (_, spilled, _) in instances.items():
        may = 0
        if kernel == "chunk_few_kernel" and args.startswith("ILi128ELb0ELb1E") and "ELi2ELi" in args:
            may = 40
        elif kernel == "chunk_kernel" and args.startswith("ILi128E"):
            may = 10
        elif (kernel, args) == ("evict_pick_kernel", "ILi32ELi1024E"):
            may = 8
        assert spilled <= may, (kernel, args, spilled)
