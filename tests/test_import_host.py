"""The binding's names and constants can be read without torch, and nothing native is loaded for them."""
import subprocess
import sys

from conftest import ROOT


def _run(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)


def test_constants_without_torch():
    code = """if True:
        import sys
        sys.modules["torch"] = None                       # an import of it raises
        import paper_1302_1690_amd
        from paper_1302_1690_amd import mpcnn
        assert (mpcnn.F32, mpcnn.BF16, mpcnn.I8, mpcnn.E4M3, mpcnn.KIND_C) == (0, 1, 2, 3, 0) and mpcnn.STATIC_WORKSPACE_BYTES > 0
        assert issubclass(mpcnn.MpcnnError, Exception) and mpcnn.SYMBOLS and mpcnn.class_beam.__doc__ and mpcnn.PackedRows.kind is not None
        assert mpcnn._lib is None and not any("libmpcnn" in line for line in open("/proc/self/maps"))
    """
    r = _run(code)
    assert r.returncode == 0, r.stderr


def test_torch_is_loaded_before_the_library():
    code = """if True:
        import sys
        from paper_1302_1690_amd import mpcnn
        assert "torch" not in sys.modules
        assert mpcnn.class_workspace_bytes(1, 8, 8, mpcnn.F32, False) > 0
        assert "torch" in sys.modules
    """
    r = _run(code)
    assert r.returncode == 0, r.stderr


def test_the_first_call_may_be_any():
    """Each in a process of its own in which nothing has loaded torch for the binding yet."""
    for call in ("mpcnn.PackedRows.empty(2, 40, mpcnn.I8, 'cpu').values", "mpcnn._dtype_of(__import__('torch').zeros(1))", "mpcnn._new((2, 3), __import__('torch').float32, 'cpu')"):
        r = _run("from paper_1302_1690_amd import mpcnn\n%s" % call)
        assert r.returncode == 0, r.stderr
