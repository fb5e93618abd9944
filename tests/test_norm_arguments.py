"""The two descriptions of the norms' argument structures in the binding agree field by field, and with the header's order."""

import ctypes
import os
import re

import pytest

from paper_2410_16135_amd import binding, build


@pytest.mark.parametrize("packed,fields,name", [
    (binding._NORM_ARGS, binding._ResidualNormArgs, "vnm_residual_norm_args"),
    (binding._NORM_BACKWARD_ARGS, binding._ResidualNormBackwardArgs, "vnm_residual_norm_backward_args")])
def test_packed_bytes_are_the_structure(packed, fields, name):
    # a value of its own for every field (exact in fp32)
    a = fields.from_buffer_copy(packed.pack(*range(1, len(fields._fields_) + 1)))
    assert [getattr(a, f) for f, _ in fields._fields_] == list(range(1, len(fields._fields_) + 1))
    header = open(os.path.join(build.ROOT, "include", "vnm.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\}" % name, header, re.S).group(1)
    declared = [(kind, f.strip(" *")) for kind, names in re.findall(r"(int64_t|int|float|const void|void)\s+([^;]+);", body)
                for f in names.split(",")]
    ctype = {"int64_t": ctypes.c_int64, "int": ctypes.c_int, "float": ctypes.c_float, "const void": ctypes.c_void_p, "void": ctypes.c_void_p}
    assert [(f, ctype[kind]) for kind, f in declared] == list(fields._fields_)
