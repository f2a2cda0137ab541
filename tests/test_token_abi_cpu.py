"""CPU-side checks of the language-model operators' entry points: what the header says and the binding says are the same, and a
NULL context is refused.  No kernel is launched here."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("gpga_embed", "gpga_embed_grad", "gpga_dropout", "gpga_layer_norm", "gpga_layer_norm_grad", "gpga_token_loss")


def test_element_types_are_those_of_the_header():
    from paper_2105_09080_amd import binding as B
    text = open(os.path.join(ROOT, "include", "gpga.h")).read()
    values = dict(re.findall(r"(GPGA_F32|GPGA_BF16|GPGA_F16) = (\d)", text))
    assert values == {"GPGA_F32": str(B.GPGA_F32), "GPGA_BF16": str(B.GPGA_BF16), "GPGA_F16": str(B.GPGA_F16)}


@pytest.mark.parametrize("name", NAMES)
def test_arguments_are_those_of_the_header(name):
    import ctypes
    from paper_2105_09080_amd import binding as B
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gpga.h")).read(), flags=re.S)
    arguments = re.search(name + r"\s*\(([^)]*)\)", text).group(1).split(",")
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "uint64_t": ctypes.c_uint64, "float": ctypes.c_float}
    want = [ctypes.c_void_p if "*" in a else kinds[a.split()[0]] for a in arguments]
    assert next(types for n, _, types in B.SIGNATURES if n == name) == want


@pytest.mark.parametrize("name", NAMES)
def test_a_null_context_is_refused(name):
    import ctypes
    from paper_2105_09080_amd import binding as B
    types = next(types for n, _, types in B.SIGNATURES if n == name)
    assert B.raw_status(name, *[None if t is ctypes.c_void_p else 0 for t in types]) == B.GPGA_EINVAL


@pytest.mark.parametrize("wide", [2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, -2 ** 32 + 5])
def test_numbers_that_do_not_fit_their_argument_are_refused(wide):
    """Cut to 32 bits a vocabulary of 2^32 + 5 would be one of 5, and layer 2^32 would have the masks of layer 0."""
    from paper_2105_09080_amd import binding as B
    calls = {"gpga_embed": (("T", "V", "D"), lambda T=1, V=1, D=1: B.gpga_embed(None, None, T, 0, V, D, 1.0, None, 1, 0)),
             "gpga_embed_grad": (("T", "V", "D"), lambda T=1, V=1, D=1: B.gpga_embed_grad(None, None, T, 0, V, D, 1.0, None, 1, 0)),
             "gpga_dropout": (("T", "D", "layer"), lambda T=1, D=1, layer=0: B.gpga_dropout(None, None, None, T, D, 1, 0, 0.1, 1, layer, None)),
             "gpga_layer_norm": (("T", "D", "layer"), lambda T=1, D=1, layer=0: B.gpga_layer_norm(
                 None, None, None, T, D, 1, 0, 0.1, 1, layer, 0, 0, 1e-5, None, None, None)),
             "gpga_layer_norm_grad": (("T", "D", "layer"), lambda T=1, D=1, layer=0: B.gpga_layer_norm_grad(
                 None, None, None, None, None, T, D, 1, 0, 0.1, 1, layer, 0, 0, None, None)),
             "gpga_token_loss": (("T", "V"), lambda T=1, V=1: B.gpga_token_loss(None, None, None, T, V, 1, 0, 1.0, None))}
    assert tuple(calls) == NAMES
    for names, call in calls.values():
        for name in names:
            with pytest.raises(B.GpgaError, match="32 bits") as e:
                call(**{name: wide})
            assert e.value.status == B.GPGA_EINVAL
            with pytest.raises(B.GpgaError) as e:                  # what fits reaches the library: no context
                call(**{name: -1})
            assert "32 bits" not in str(e.value) and e.value.status == B.GPGA_EINVAL
