"""The check of the AdamW step's kind of rounding: synchronous, before anything touches a device."""
import ctypes

import pytest

import paper_1906_03707_b200 as hb
from paper_1906_03707_b200.build import build as build_library


@pytest.mark.parametrize("rounding,status", [(hb.HAG_NEAREST, 0), (hb.HAG_CHANCE, 0), (2, hb.HAG_ERR_ARG), (-1, hb.HAG_ERR_ARG)])
@pytest.mark.parametrize("kind", [hb.HAG_STATE32, hb.HAG_STATE8])
def test_rounding(rounding, status, kind):
    build_library()
    o = hb.HagAdamwOptions(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, seed=3, rounding=rounding)
    assert hb.load_library().hag_adamw_step(0, None, None, None, None, None, None, None, kind, None, None, None, ctypes.byref(o), None) == status


def test_options_have_the_headers_fields():
    import os
    import re
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hag.h")).read()
    body = re.search(r"typedef struct hag_adamw_options \{(.*?)\}", header, re.S).group(1)
    names = [n.strip(" *") for line in body.split(";") if line.strip() for n in re.sub(r"^\s*(const )?\w+ ", "", line).split(",")]
    assert names == [f[0] for f in hb.HagAdamwOptions._fields_]
