"""Loading the library: one that is older than the binding is told of as such, and there is one HIP runtime in the process."""
import os
import subprocess
import sys

import pytest


def older(tmp_path, version, exports):
    src, so = tmp_path / "old.c", tmp_path / "librkc.so"
    src.write_text(f"int rkc_abi_version(void) {{ return {version}; }}\n" + "".join(f"int {n}(void) {{ return 0; }}\n" for n in exports if n != "rkc_abi_version"))
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", str(so), str(src)])
    return str(so)


@pytest.mark.parametrize("what", ["replay alone", "no rows", "the version alone"])
@pytest.mark.parametrize("version", [4, 5])
def test_an_older_library_is_to_be_rebuilt(tmp_path, monkeypatch, version, what):
    """Of another ABI, and of this one before functions were added: both say what to do, and nothing is kept."""
    import paper_2605_24259_amd as rkc
    exports = rkc.EXPORTS + (rkc.cache.CACHE_EXPORTS if what == "no rows" else ())
    path = older(tmp_path, version, exports if what != "the version alone" else ())
    monkeypatch.setattr(rkc, "LIB_PATH", path)
    monkeypatch.setattr(rkc, "_lib", None)
    with pytest.raises(RuntimeError, match="rebuild the library") as e:
        rkc.load()
    assert path in str(e.value) and rkc._lib is None
    assert ("ABI 4" in str(e.value)) == (version == 4) and ("lacks rkc_" in str(e.value)) == (version == 5)


def test_one_hip_runtime_whatever_comes_first():
    """The library takes the HIP runtime that torch brings, also where it is loaded before torch: with two in the process, streams
    and memory of the one mean nothing to the other."""
    code = ("import paper_2605_24259_amd as rkc\nrkc.load()\nimport torch\n"
            "print(len({x.split()[-1] for x in open('/proc/self/maps') if 'libamdhip64' in x}))")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert subprocess.check_output([sys.executable, "-c", code], text=True, cwd=root).strip() == "1"
