"""Compile the gfx950 HIP library libsd2.so in-tree (hipcc, no JIT cache), and the binding of its paged calls to torch
tensors (_torch_paged.so: host code only)."""
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
SO = os.path.join(HERE, "libsd2.so")
TORCH_SO = os.path.join(HERE, "_torch_paged.so")
SOURCES = ["csrc/kernels.hip", "csrc/wsgemv.hip", "csrc/pgemm.hip", "csrc/attn.hip", "csrc/mk.hip", "csrc/engine.hip",
           "csrc/paged_attn.hip", "csrc/paged_attn_window.hip", "csrc/paged_attn_scaled_bf16.hip",
           "csrc/paged_attn_scaled_f32.hip", "csrc/paged_append8.hip", "csrc/pages.hip"]
# XNACK off: MI355X runs with page-fault replay disabled by default, and code built for that
# mode forms longer load clauses than the "any" target (0.9 % less time per round measured)
ARCH = "gfx950:xnack-"


def hipcc() -> str:
    p = shutil.which("hipcc")
    if p:
        return p
    p = "/opt/rocm/bin/hipcc"
    if os.path.exists(p):
        return p
    raise RuntimeError("hipcc not found: the SD2 library needs ROCm's hipcc to build")


FLAGS = ["-O3", "-std=c++17", "-fPIC",
         # packed fp32 instructions are kept out of every kernel
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall"]


def build(verbose: bool = False) -> str:
    """Compile every source to an object in parallel (each object carries its own gfx950 code
    object; no relocatable device code is needed), then link the shared library, and the binding against it."""
    from concurrent.futures import ThreadPoolExecutor

    import torch
    torch_dir = os.path.dirname(torch.__file__)

    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    cc = hipcc()

    def compile_one(src):
        obj = os.path.join(objdir, os.path.basename(src).replace(".hip", ".o"))
        cmd = [cc, f"--offload-arch={ARCH}", *FLAGS, "-c", "-o", obj, os.path.join(HERE, src)]
        return obj, subprocess.run(cmd, capture_output=True, text=True)

    def compile_binding():
        obj = os.path.join(objdir, "torch_paged.o")
        include = os.path.join(torch_dir, "include")
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
               "-isystem", include, "-isystem", os.path.join(include, "torch/csrc/api/include"),
               "-isystem", sysconfig.get_paths()["include"], "-c", "-o", obj, os.path.join(HERE, "csrc/torch_paged.cpp")]
        return obj, subprocess.run(cmd, capture_output=True, text=True)

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        binding = ex.submit(compile_binding)
        results = list(ex.map(compile_one, SOURCES))
        binding_obj, binding_res = binding.result()
    msgs = []
    for (obj, res), src in zip(results, SOURCES):
        if res.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n" + res.stderr)
        msgs += [l for l in res.stderr.splitlines() if "packed-fp32-ops' is not a recognized" not in l]
    link = [cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", SO + ".tmp"] + [o for o, _ in results]
    res = subprocess.run(link, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stderr)
    if verbose and msgs:
        print("\n".join(msgs))
    os.replace(SO + ".tmp", SO)
    if binding_res.returncode != 0:
        raise RuntimeError("g++ failed on csrc/torch_paged.cpp:\n" + binding_res.stderr)
    # torch's libraries are those that `import torch` has loaded by the time the binding is
    res = subprocess.run(["g++", "-shared", "-o", TORCH_SO + ".tmp", binding_obj, "-L" + HERE, "-l:libsd2.so",
                          "-L" + os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN"],
                         capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("linking the binding failed:\n" + res.stderr)
    os.replace(TORCH_SO + ".tmp", TORCH_SO)
    return SO


if __name__ == "__main__":
    print(build(verbose=True))
