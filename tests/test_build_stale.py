"""When the library is compiled again: any of its sources or headers is newer than it."""
from __future__ import annotations

import os

import pytest

from paper_2608_12574_gb300 import _build

NAMES = sorted(n for n in os.listdir(_build.CSRC)) + sorted(os.path.join("include", n) for n in os.listdir(_build.INCLUDE))


@pytest.mark.parametrize("changed", NAMES)
def test_newer_source(changed, tmp_path, monkeypatch):
    paths = {n: tmp_path / ("inc" if os.path.dirname(n) else "src") / os.path.basename(n) for n in NAMES}
    for path in paths.values():
        path.parent.mkdir(exist_ok=True)
        path.write_text("")
        os.utime(path, (100, 100))
    lib = tmp_path / "lib.so"
    monkeypatch.setattr(_build, "CSRC", str(tmp_path / "src"))
    monkeypatch.setattr(_build, "INCLUDE", str(tmp_path / "inc"))
    monkeypatch.setattr(_build, "LIB", str(lib))
    assert _build._stale()
    lib.write_text("")
    os.utime(lib, (200, 200))
    assert not _build._stale()
    os.utime(paths[changed], (300, 300))
    assert _build._stale()
