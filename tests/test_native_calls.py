"""The native binding offers what is called through it, and nothing else."""
import glob
import os

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_native_function_is_called():
    from paper_1802_00150_b200 import amq
    text = ""
    for path in glob.glob(os.path.join(ROOT, "paper_1802_00150_b200", "*.py")) + glob.glob(os.path.join(ROOT, "tests", "*.py")):
        with open(path) as f:
            text += f.read()
    for name in dir(amq._native):
        if not name.startswith("_"):
            assert "_native.%s(" % name in text, name
