"""What is built for whom: the C-ABI library without torch's headers, the extension anew for another Python or torch."""
import subprocess
import sys

from paper_2608_21614_b200 import build


def test_the_extension_is_built_for_this_python_and_torch(monkeypatch):
    from paper_2608_21614_b200 import mx                                # noqa: F401  (builds it)
    assert not build.host_stale()
    version = build.importlib.metadata.version
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "9.9.9" if name == "torch" else version(name))
    assert build.host_stale()
    monkeypatch.undo()
    monkeypatch.setattr(build.sysconfig, "get_config_var", lambda name: "cpython-399")
    assert build.host_stale()
    monkeypatch.undo()
    assert not build.host_stale()


def test_the_older_entry_points_do_not_need_the_extension():
    """binding and layer load with no compiler for the extension and no extension there."""
    program = ("from paper_2608_21614_b200 import build\n"
               "build.HOST_LIB = build.HOST_LIB + '.missing'\n"
               "def refuse(*a, **k): raise RuntimeError('the extension was asked for')\n"
               "build.build_host_calls = refuse\n"
               "from paper_2608_21614_b200 import binding, layer, stack\n"
               "assert binding.saem_version() >= 100\n"
               "try:\n"
               "    from paper_2608_21614_b200 import mx\n"
               "except RuntimeError as e:\n"
               "    print(e)\n")
    r = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, cwd=build._ROOT)
    assert r.returncode == 0 and r.stdout.strip() == "the extension was asked for", r.stderr


def test_the_extension_can_be_imported_by_its_name_first():
    r = subprocess.run([sys.executable, "-c", "from paper_2608_21614_b200 import _host_calls as c; print(c.quantize.__name__)"], capture_output=True,
                       text=True, cwd=build._ROOT)
    assert r.returncode == 0 and r.stdout.strip() == "quantize", r.stderr
