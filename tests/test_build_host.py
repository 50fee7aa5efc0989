"""What the build makes of the compiled part of the binding."""

import os
import sysconfig

from paper_2605_28803_gb300 import build, qvla

SUFFIX = sysconfig.get_config_var("EXT_SUFFIX")


def test_the_compiled_calls_are_this_interpreters():
    """Named with the interpreter's tag, so that another one neither imports them nor takes them for its own."""
    assert os.path.basename(qvla._calls.__file__) == "_calls" + SUFFIX
    assert build.CALLS == qvla._calls.__file__
    assert not os.path.exists(os.path.join(build.PKG, "_calls.so"))  # (a file without a tag serves every interpreter)


def test_calls_of_another_interpreter_do_not_count_as_built():
    other = build.CALLS.replace(SUFFIX, ".cpython-399-" + SUFFIX.split("-", 2)[2])
    assert other != build.CALLS and build._stale(other)
