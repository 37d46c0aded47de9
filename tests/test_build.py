"""What the build makes, and what it needs for it."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_library_is_built_without_torch(tmp_path):
    """A C user needs nvcc alone: with torch not importable the library is linked all the same, and the marshalling
    module (whose place is empty here) left out."""
    from paper_2511_06010_b200 import build

    build.build()
    program = ("import sys; sys.modules['torch'] = None\n"
               "from paper_2511_06010_b200 import build as b\n"
               f"b.LIB = {str(tmp_path / 'libmoska.so')!r}; b.CALL = {str(tmp_path / '_paged_call.so')!r}\n"
               "print(b.build())")
    r = subprocess.run([sys.executable, "-c", program], cwd=ROOT, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stderr
    assert r.stdout.strip() == str(tmp_path / "libmoska.so") and os.listdir(tmp_path) == ["libmoska.so"]


def test_a_module_built_for_another_torch_is_refused_and_built_again():
    from paper_2511_06010_b200 import build

    build.build()
    program = ("import torch\n"
               "torch.__version__ = '0.0'\n"
               "from paper_2511_06010_b200 import build as b\n"
               "b.os.replace = lambda *a: b.os.remove(a[0])\n"   # what it would build is thrown away
               "made = []\n"
               "b.subprocess.check_call = lambda c, **k: (made.append(c), open(c[c.index('-o') + 1], 'w').close())\n"
               "b.build_call()\n"
               "assert len(made) == 1, 'not built again'\n"
               "try:\n"
               "    import paper_2511_06010_b200.paged\n"
               "except ImportError as e:\n"
               "    assert 'build it again' in str(e), e\n"
               "else:\n"
               "    raise SystemExit('imported')\n")
    r = subprocess.run([sys.executable, "-c", program], cwd=ROOT, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stderr + r.stdout
