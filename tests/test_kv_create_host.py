"""What making a handle of the KV-cache operators does and leaves to later calls, from the source (no GPU)."""

import os
import re

KV = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_12659_gb300", "csrc", "kv")


def function(name, start):
    with open(os.path.join(KV, name)) as f:
        text = f.read()
    text = text[text.index(start):]
    return text[:text.index("\n}\n")]


def test_kernels_over_windows_and_8_bit_caches_are_looked_up_by_the_first_call_of_them():
    assert "kv_span" not in function("kv_api.cu", "JPI_API jpi_status jpi_kv_create(")
    launch = function("kv_span.cu", "jpi_status launch_kv_span(")
    assert re.search(r"if \(!h->span_ready\) JPI_TRY\(kv_span_prepare\(h\)\);", launch)
    # Only a look-up that went through is not made again.
    prepare = function("kv_span.cu", "jpi_status kv_span_prepare(")
    assert prepare.rindex("h->span_ready = true;") > prepare.rindex("JPI_TRY(") and prepare.rstrip().endswith("return JPI_OK;")
