"""_seq.so, which puts the sequence operators behind Python: only they need it, and it is built anew for another torch or Python (no GPU)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(body):
    r = subprocess.run([sys.executable, "-c", "import paper_2407_16990_amd as pkg\nfrom paper_2407_16990_amd import binding, build\nimport pytest, torch\n" + body + "\nprint('DONE')"],
                       capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0 and r.stdout.strip().endswith("DONE"), r.stdout[-2000:] + r.stderr[-3000:]


def test_the_image_path_loads_without_it():
    """No module, and no host compiler to build it: the library loads and works, and a sequence operator says what is missing."""
    _run('''
import os
os.environ["CXX"] = "/no/such/compiler"
build.MODULE, build.MODULE_STAMP = "/nowhere/_seq.so", "/nowhere/_seq.so.sources"
lib = pkg.load_library()
import workloads as wl
assert lib.rh_budget(96, 96, 3) > 0 and len(pkg.needed_radii(wl.Net("edsr", 64, 1, 2))) > 0
with pytest.raises(OSError, match="compiler"):
    pkg.KVCache(*[torch.zeros(1, 1, 1, 32)] * 2)
''')


def test_another_torch_or_python_makes_it_stale():
    _run('''
import shutil, sys, tempfile
build.build_module()
assert not build.module_is_stale()
here = tempfile.mkdtemp()
for name in ("MODULE", "MODULE_STAMP"):
    old = getattr(build, name)
    setattr(build, name, shutil.copy(old, here))
assert not build.module_is_stale()
version = torch.__version__
torch.__version__ = "0.0.1"
assert build.module_is_stale()
torch.__version__ = version
with open(build.MODULE_STAMP) as f: good = f.read()
with open(build.MODULE_STAMP, "w") as f: f.write("made for another\\n")
assert build.module_is_stale()
# and the first operator that is called builds it again
calls = []
def build_module(force=False):
    calls.append(force)
    with open(build.MODULE_STAMP, "w") as f: f.write(good)
build.build_module = build_module
binding._seq.matvec_packed
assert len(calls) == 1
binding._seq.norm_residual
assert len(calls) == 1 and not build.module_is_stale()
shutil.rmtree(here)
''')


def test_the_library_alone_is_not_built_for_the_module():
    _run('''
build.source_digest(), build.module_digest()
seen = []
build._digest = lambda paths, extra="": seen.append([p.rsplit("/", 1)[-1] for p in paths]) or "x"
build.source_digest()
assert build.MODULE_SOURCE not in seen[0] and "seq_matvec.hip" in seen[0]
build.module_digest()
assert build.MODULE_SOURCE in seen[1] and "rh_seq.h" in seen[1]
''')
