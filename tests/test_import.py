"""What importing the binding costs."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_binding_is_imported_without_torch():
    """Callers of the entry points that take numpy arrays do not pay for it."""
    code = "import sys; from paper_2511_13732_b200 import binding; binding.load(); assert 'torch' not in sys.modules"
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ROOT)
