"""The module that marshals the paged-cache calls belongs to one interpreter: its file is named for it, another one's is
neither loaded nor taken as built."""
import os
import sysconfig

import pytest

import paper_2607_02501_gb300 as emb
from paper_2607_02501_gb300 import buildlib

SUFFIX = sysconfig.get_config_var("EXT_SUFFIX")


def test_module_is_this_interpreter_s():
    emb.build()
    m = emb._binding()
    assert m.__file__.endswith("_paged_binding" + SUFFIX) and os.path.samefile(m.__file__, buildlib.BINDING)


def test_another_interpreter_s_is_not_taken_for_it(monkeypatch):
    emb.build()
    assert not buildlib._stale()
    monkeypatch.setattr(buildlib, "BINDING", buildlib.BINDING.replace(SUFFIX, ".cpython-399-none.so"))
    monkeypatch.setattr(emb, "_marshal", None)
    assert buildlib._stale()
    with pytest.raises(RuntimeError, match="with this interpreter"):
        emb._binding()
