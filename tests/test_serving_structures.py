"""The ctypes structures of the batched decoding calls name the C header's fields, in its
order and of its types (the compiled binding is built from the header itself)."""
import ctypes as C
import os
import re

import pytest

from paper_2608_15383_amd import _lib

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "exactmoe_serving.h")
SCALARS = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}


def fields(name):
    """[(field, ctypes type)] of a structure of the header."""
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, re.S).group(1)
    out = []
    for line in filter(None, (d.strip() for d in body.split(";"))):
        kind, names = re.match(r"(?:const\s+)?(\w+)\s*(.*)", line, re.S).groups()
        for n in names.split(","):
            pointer, n = "*" in n, n.replace("*", "").strip()
            out.append((n, C.c_void_p if pointer else SCALARS[kind]))
    return out


@pytest.mark.parametrize("name,view", [
    ("emoe_paged_kv", _lib.PagedKVView), ("emoe_paged_append_args", _lib.PagedAppendArgs),
    ("emoe_paged_attention_args", _lib.PagedAttentionArgs), ("emoe_logits_args", _lib.LogitsArgs),
    ("emoe_decoder_batch", _lib.DecoderBatch)])
def test_fields(name, view):
    assert [tuple(f) for f in view._fields_] == fields(name)
