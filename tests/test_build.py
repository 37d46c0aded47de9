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
