"""What has to be built for what: the C library alone for its callers, the torch extension for the calls on tensors, one per
version of torch."""
import os
import shutil
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import paper_2501_05370_b200 as sds
assert sds.load().sds_strerror(0) and sds.gated_ffn_bytes(4, 64, 128).keep_bytes > 0
import torch
for again in range(2):
    try:
        sds.layer_norm(torch.zeros(2, 8))
    except RuntimeError as e:
        assert "no-such-compiler" in str(e) and "torch extension" in str(e), e
    else:
        raise AssertionError("a call on tensors without the extension")
print("loaded")
"""


def test_the_library_loads_without_the_extension_and_without_compilers(tmp_path):
    import paper_2501_05370_b200 as sds
    sds.load()
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    shutil.copytree(os.path.join(ROOT, "paper_2501_05370_b200"), tmp_path / "paper_2501_05370_b200",
                    ignore=shutil.ignore_patterns("_sds_torch*", "_build", "__pycache__"))
    env = dict(os.environ, CXX="no-such-compiler", NVCC="no-such-nvcc")
    r = subprocess.run([sys.executable, "-c", CODE], cwd=tmp_path, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "loaded" in r.stdout, r.stdout + r.stderr


def test_the_extension_is_of_one_version_of_torch(monkeypatch):
    import torch
    from paper_2501_05370_b200 import build, layers
    if build.needs_ext_build():
        build.build()
    assert not build.needs_ext_build() and torch.__version__ in os.path.basename(build.ext_path())
    assert os.path.samefile(layers._ext().__file__, build.ext_path())
    monkeypatch.setattr(torch, "__version__", torch.__version__ + ".later")
    assert build.needs_ext_build() and not build.needs_build()
