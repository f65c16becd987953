"""The library without its native short forms: a compiler, a file or a torch that does not suit
costs the short calls some host time and nothing else (no GPU needed)."""
import os
import re
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

import paper_2609_30846_gb300 as ip
from paper_2609_30846_gb300 import _build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(autouse=True)
def with_torch():
    ip.build()
    if _build._torch_dir() is None:
        pytest.skip("no torch with CUDA to build for")


@pytest.fixture
def fresh(monkeypatch):
    """The binding as before its first call."""
    monkeypatch.setattr(ip, "_lib", None)
    monkeypatch.setattr(ip, "_short", ip._Unbound)


def works():
    """Calls of both kinds answer, by the general forms."""
    assert ip._short is ip._Unbound
    assert ip.workspace_bytes(1, 8, 64) == 256
    assert ip.dyadic_multiplier(0.5)
    with pytest.raises(TypeError, match="CUDA tensor"):
        ip.quantize_rows_i8(torch.zeros(2, 16))


@pytest.mark.parametrize("what", ["missing", "garbage", "other module"])
def test_a_file_that_does_not_load(fresh, monkeypatch, tmp_path, what):
    path = tmp_path / "ip_torch.so"
    if what == "garbage":
        path.write_bytes(b"\x7fELF" + bytes(200))
    elif what == "other module":
        (tmp_path / "m.c").write_text("int nothing;")
        subprocess.run([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-o", str(path), str(tmp_path / "m.c")], check=True)
    monkeypatch.setattr(_build, "torch_extension", lambda: str(path))
    with pytest.warns(RuntimeWarning, match="short forms"):
        ip.load(build_if_missing=False)
    works()


@pytest.mark.parametrize("cmd", [["false"], ["/nonexistent/compiler"], None])
def test_a_compiler_that_fails(fresh, monkeypatch, tmp_path, cmd):
    path = str(tmp_path / "ip_torch.so")
    monkeypatch.setattr(_build, "torch_extension", lambda: path)

    def command(out):
        if cmd is None:
            raise RuntimeError("no headers")
        return cmd
    monkeypatch.setattr(_build, "torch_command", command)
    before = os.path.getmtime(_build.LIB)
    with pytest.warns(RuntimeWarning, match="short forms"):
        assert ip.build() == _build.LIB
    assert os.path.getmtime(_build.LIB) == before and os.listdir(tmp_path) == []      # the library is not built again
    with pytest.warns(RuntimeWarning, match="short forms"):
        ip.load()
    works()


def test_a_torch_that_is_not_as_expected(fresh, monkeypatch):
    def odd():
        raise OSError("no version.py")
    monkeypatch.setattr(_build, "_torch_version", odd)
    with pytest.warns(RuntimeWarning, match="short forms"):
        ip.load()
    works()


def test_the_versions_are_part_of_the_name(monkeypatch):
    path = _build.torch_extension()
    assert torch.__version__ in path and _build.up_to_date() and os.path.exists(path)
    assert re.search(r"%d%d" % sys.version_info[:2], os.path.basename(path))
    monkeypatch.setattr(_build, "_torch_version", lambda: "1.2.3")
    assert _build.torch_extension() != path and not _build.up_to_date()


def test_a_library_built_before_these_calls(fresh, monkeypatch, tmp_path):
    later = [n for n in ip.EXPORTS if n.startswith(("ip_quantize_rows", "ip_linear_scaled", "ip_kv4"))]
    assert len(later) == 7
    src = "".join(f"int {n}(void) {{ return 0; }}\n" for n in ip.EXPORTS if n not in later)
    (tmp_path / "old.c").write_text(src)
    old = str(tmp_path / "old.so")
    subprocess.run([os.environ.get("CC", "gcc"), "-shared", "-fPIC", "-o", old, str(tmp_path / "old.c")], check=True)
    monkeypatch.setattr(_build, "LIB", old)
    with pytest.warns(RuntimeWarning, match="short forms"):
        lib = ip.load(build_if_missing=False)
    assert lib.ip_debug_set_split_mode(-1) == 0 and ip._short is ip._Unbound
    with pytest.raises(AttributeError, match="ip_kv4_page_bytes"):
        ip.kv4_page_bytes(16)
