"""Build ``libqsdp.so`` (HIP kernels + C ABI) for gfx950 with hipcc, in-tree.

``python -m paper_2302_02390_amd.build`` compiles every translation unit (in parallel) and
links ``paper_2302_02390_amd/libqsdp.so``. Flags: strict binary32 arithmetic (no contraction, no
reassociation, no reciprocal or other approximations: ``-fno-fast-math``), with ONE relaxation,
``-fno-honor-nans``: inputs are finite by contract, so ``fminf``/``fmaxf`` may compile to single
``v_min``/``v_max`` instructions instead of NaN-canonicalising sequences (measured on the 1.3B
vector: quantize_grad 0.97 ms with the flag, 1.05 ms without; the code-resident step 1.43 against
1.55 ms). The flag changes no result for finite inputs. Packed-fp32 instruction selection is
switched off.
"""
import glob
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libqsdp.so")
BENCH_LIB = os.path.join(HERE, "libqsdp_bench.so")  # streaming kernels for bench.py, not part of the codec

# The binding's argument marshalling: a Python extension module, so its name says which interpreter it is for.
MARSHAL = os.path.join(HERE, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-fno-fast-math", "-fno-honor-nans", "-Wall", "-Wno-unused-result",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"] + os.environ.get("QSDP_EXTRA_FLAGS", "").split()

# bucket size -> (lanes per bucket G, rows per wave R, waves per bucket W): bucket = 4 * G * R * W
WAVE_SHAPES = {128: (8, 4, 1), 256: (16, 4, 1), 512: (32, 4, 1), 1024: (64, 4, 1), 2048: (64, 4, 2),
               4096: (64, 4, 4)}
# team shapes of the tile kernel, which serves every other bucket size: (waves, rows)
TILE_SHAPES = [(1, 2), (4, 2), (1, 4), (1, 6), (1, 8), (4, 4), (4, 6), (4, 8)]
# shapes of the level fit: (values per lane, waves per batch), for buckets of up to 64 * values * waves
FIT_SHAPES = [(2, 1), (4, 1), (8, 1), (16, 1), (32, 1), (16, 4), (16, 8)]

# the operators on logits and on packed weights (csrc/lm): masks are infinities there, and a NaN has to come through
LM_FLAGS = ["-fhonor-nans"]
# the kernels on rows of logits, one object for each format of theirs (lm_common.hpp)
LM_FORMATS = ["F32", "BF16", "F16"]


def _units():
    # the longest compiles first: with all formats in one object, and that the last, eight jobs took 252 s instead of 110
    units = [(f"lm_rows_{t.lower()}.o", os.path.join("lm", "lm_rows.hip"), LM_FLAGS + [f"-DQSDP_LM_FORMAT={t}"])
             for t in LM_FORMATS]
    units += [(f"{name}.o", os.path.join("lm", f"{name}.hip"), LM_FLAGS) for name in ("lm_linear", "lm_api")]
    units.append(("qsdp_api.o", "qsdp_api.hip", []))
    for b, (g, r, w) in WAVE_SHAPES.items():
        units.append((f"qsdp_wave_{b}.o", "qsdp_wave_inst.hip",
                      [f"-DQSDP_G={g}", f"-DQSDP_R={r}", f"-DQSDP_W={w}", f"-DQSDP_B={b}"]))
    # the weight quantizer alone also as two waves per 1024-bucket (its faster shape; the other modes are not)
    units.append(("qsdp_wave_1024w2.o", "qsdp_wave_inst.hip",
                  ["-DQSDP_G=64", "-DQSDP_R=2", "-DQSDP_W=2", "-DQSDP_B=1024", "-DQSDP_WEIGHT_ONLY=1024w2"]))
    for w, r in TILE_SHAPES:
        units.append((f"qsdp_tile_{w}_{r}.o", "qsdp_tile_inst.hip", [f"-DQSDP_TILE_W={w}", f"-DQSDP_TILE_R={r}"]))
    for v, w in FIT_SHAPES:
        units.append((f"qsdp_fit_{v}_{w}.o", "qsdp_fit_inst.hip", [f"-DQSDP_FIT_V={v}", f"-DQSDP_FIT_W={w}"]))
    return units


def _compile(unit):
    obj, src, defs = unit
    out = os.path.join(OBJ, obj)
    cmd = [HIPCC] + FLAGS + defs + ["-c", os.path.join(CSRC, src), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return out


def build(jobs=None, verbose=False):
    os.makedirs(OBJ, exist_ok=True)
    jobs = jobs or min(8, os.cpu_count() or 1)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(_compile, _units()))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    if verbose:
        print(LIB)
    try:
        build_marshal(verbose)
    except (ImportError, OSError, RuntimeError) as e:  # no torch, no g++, no headers, or others than it was written for
        print(f"the binding's argument marshalling is not built, its Python functions do that work: {e}", file=sys.stderr)
    build_bench_support(verbose)
    return LIB


def build_marshal(verbose=False):
    """The binding's argument marshalling (csrc/qsdp_marshal.cpp, host code against torch's headers). The library and
    programs in C need neither it nor torch."""
    for old in glob.glob(os.path.join(HERE, "_marshal*.so")):  # none of another library or torch stays behind
        os.remove(old)
    import torch
    from torch.utils import cpp_extension
    includes = [sysconfig.get_paths()["include"]] + cpp_extension.include_paths("cuda")
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", "-Wall", "-D__HIP_PLATFORM_AMD__",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DQSDP_TORCH_VERSION="{torch.__version__} {torch.version.git_version}"']
    for d in includes:
        cmd += ["-isystem", d]
    cmd += [os.path.join(CSRC, "qsdp_marshal.cpp"), "-o", MARSHAL, "-L", HERE, "-lqsdp"]
    for d in cpp_extension.library_paths("cuda"):
        cmd += ["-L", d]
    cmd += ["-ltorch_python", "-ltorch_cpu", "-lc10", "-lamdhip64", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    if verbose:
        print(MARSHAL)
    return MARSHAL


def build_bench_support(verbose=False):
    """libqsdp_bench.so: the plain streaming kernels bench.py times beside the codec (csrc/qsdp_bench_stream.hip)."""
    cmd = [HIPCC] + FLAGS + ["-shared", os.path.join(CSRC, "qsdp_bench_stream.hip"), "-o", BENCH_LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    if verbose:
        print(BENCH_LIB)
    return BENCH_LIB


def build_client(verbose=False):
    """The plain C example client (examples/qsdp_client.c) against the built library, with gcc."""
    root = os.path.dirname(HERE)
    src = os.path.join(root, "examples", "qsdp_client.c")
    out = os.path.join(root, "examples", "qsdp_client")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    cmd = ["gcc", "-std=c11", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"),
           "-I", os.path.join(rocm, "include"), src, "-L", HERE, "-lqsdp", "-L", os.path.join(rocm, "lib"),
           "-lamdhip64", "-Wl,-rpath,$ORIGIN/../paper_2302_02390_amd", "-Wl,-rpath," + os.path.join(rocm, "lib"),
           "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    if verbose:
        print(out)
    return out


if __name__ == "__main__":
    build(verbose=True)
    build_client(verbose=True)
    sys.exit(0)
