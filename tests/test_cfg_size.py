"""A program and a library that disagree about epikv_cfg's size can tell."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_and_binding_agree_with_the_header():
    from paper_2606_26472_amd import epikv as E
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "epikv.h")).read(), flags=re.S)
    body = re.search(r"typedef struct epikv_cfg \{(.*?)\} epikv_cfg;", text, re.S).group(1)
    names = re.findall(r"(\w+)\s*;", body)
    assert [f[0] for f in E.Cfg._fields_] == names  # (all of 4 bytes)
    assert E.lib().epikv_cfg_bytes() == ctypes.sizeof(E.Cfg) == 4 * len(names)


@pytest.mark.parametrize("nbytes", [0, 60, 68])
def test_the_binding_refuses_another_size(nbytes):
    from paper_2606_26472_amd import epikv as E
    E._same_cfg(ctypes.sizeof(E.Cfg))
    assert nbytes != ctypes.sizeof(E.Cfg)
    with pytest.raises(RuntimeError, match="build the library anew"):
        E._same_cfg(nbytes)
