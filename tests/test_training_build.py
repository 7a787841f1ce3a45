"""What the compiler made of the kernels of a training step (no GPU needed: hipcc cross-compiles gfx950): no scratch memory for those that carry
the time, and the registers and LDS that the workgroups on a compute unit were counted with."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2205_09707_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

# part of the mangled name -> (source, most vector registers, most LDS bytes)
KERNELS = {
    "loss_mm_kernelILi0ELi0E": ("k_loss_mm", 256, 160 << 10),      # eight waves, two per SIMD, one workgroup per CU
    "loss_mm_kernelILi1ELi1E": ("k_loss_mm", 256, 160 << 10),
    "loss_gradients_kernelILi0E": ("k_loss_mm", 256, 160 << 10),
    "loss_few_kernelILi0ELi4ELi1ELi1ELb0E": ("k_loss", 64, 32 << 10),   # five workgroups per CU
    "loss_few_kernelILi0ELi4ELi1ELi3ELb0E": ("k_loss", 64, 53 << 10),   # three
    "loss_few_kernelILi0ELi4ELi1ELi8ELb0E": ("k_loss", 256, 80 << 10),  # two, a wave of each per SIMD
    "loss_few_kernelILi0ELi8ELi2ELi8ELb0E": ("k_loss", 256, 160 << 10),
    "norm_kernelILi0ELi64ELi4E": ("k_norm", 128, 1 << 10),
    "norm_grad_kernelILi0ELi256ELi1E": ("k_norm", 102, 1 << 10),        # five waves per SIMD
    "norm_grad_kernelILi0ELi256ELi4E": ("k_norm", 256, 1 << 10),
    "dropout_kernelILi0ELb1E": ("k_dropout", 64, 0),                    # eight
    "embed_kernelILi0ELi4E": ("k_embed", 64, 0),
    "embed_grad_kernelILi0ELb1E": ("k_embed", 80, 0),                   # six
}


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    if not (os.path.exists(HIPCC) or shutil.which(HIPCC)):
        pytest.skip("no hipcc")
    out = {}
    for source in sorted({s for s, _, _ in KERNELS.values()}):
        path = tmp_path_factory.mktemp("asm") / (source + ".asm")
        cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I" + os.path.join(ROOT, "include"),
               "-I" + CSRC, "--cuda-device-only", "-S", os.path.join(CSRC, source + ".hip"), "-o", str(path)]
        r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout
        out[source] = path.read_text()
    return out


@pytest.mark.parametrize("name", KERNELS)
def test_registers_and_lds(assembly, name):
    source, registers, lds = KERNELS[name]
    found = [b for b in re.split(r"\n  - ", assembly[source][assembly[source].index("amdhsa.kernels:"):]) if re.search(r"\.symbol:\s+\S*" + name, b)]
    assert len(found) == 1, name
    value = lambda key: int(re.search(r"\." + key + r":\s+(\d+)", found[0]).group(1))  # noqa: E731
    assert value("private_segment_fixed_size") == 0 and value("vgpr_spill_count") == 0
    assert value("vgpr_count") <= registers
    assert value("group_segment_fixed_size") <= lds
