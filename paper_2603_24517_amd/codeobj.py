"""Reads the gfx950 code objects inside a library built here: the metadata notes (register counts, scratch size, spills per
kernel) and the instructions, for checks of waits that the compiler does not make."""
import os
import re
import subprocess
import tempfile

LLVM_BIN = os.environ.get("ROCM_LLVM_BIN", "/opt/rocm/llvm/bin")
TARGET = "hipv4-amdgcn-amd-amdhsa--gfx950"
FIELDS = ("vgpr_count", "agpr_count", "sgpr_count", "vgpr_spill_count", "sgpr_spill_count",
          "private_segment_fixed_size", "group_segment_fixed_size", "max_flat_workgroup_size")


def _bundles(fatbin):
    """The bundles of a library's section: one for each translation unit with device code."""
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    starts = [m.start() for m in re.finditer(magic, fatbin)]
    return [fatbin[a:b] for a, b in zip(starts, starts[1:] + [len(fatbin)])]


def _read(lib_path, *tool):
    """What an LLVM tool prints for every gfx950 code object of the library."""
    text = ""
    with tempfile.TemporaryDirectory() as tmp:
        fatbin, part, code = (os.path.join(tmp, n) for n in ("fatbin", "part", "code.o"))
        subprocess.run([os.path.join(LLVM_BIN, "llvm-objcopy"), "-O", "binary", "--only-section=.hip_fatbin",
                        lib_path, fatbin], check=True)
        with open(fatbin, "rb") as f:
            bundles = _bundles(f.read())
        for bundle in bundles:
            with open(part, "wb") as f:
                f.write(bundle)
            subprocess.run([os.path.join(LLVM_BIN, "clang-offload-bundler"), "--unbundle", "--type=o",
                            f"--targets={TARGET}", f"--input={part}", f"--output={code}"], check=True)
            text += subprocess.run([os.path.join(LLVM_BIN, tool[0]), *tool[1:], code], check=True, capture_output=True, text=True).stdout
    return text


def disassembly(lib_path):
    """The instructions of every kernel of the library, in order, one "name operands" each."""
    lines = []
    for line in _read(lib_path, "llvm-objdump", "-d", "--no-show-raw-insn").splitlines():
        text = line.split("//")[0].split(";")[0].strip()
        if line[:1].isspace() and text:
            lines.append(" ".join(text.split()))
    return lines


def kernel_metadata(lib_path):
    """{kernel symbol: {field: int}} for every kernel of the library's gfx950 code objects."""
    notes = _read(lib_path, "llvm-readelf", "--notes")
    kernels = {}
    for entry in re.split(r"\n\s*- \.", notes):
        name = re.search(r"\.name:\s+(\S+)", entry)
        if not name or ".vgpr_count" not in entry and "vgpr_count" not in entry:
            continue
        fields = {}
        for f in FIELDS:
            m = re.search(r"\.?%s:\s+(\d+)" % f, entry)
            if m:
                fields[f] = int(m.group(1))
        if "vgpr_count" in fields:
            kernels[name.group(1)] = fields
    return kernels
