"""The rollout binding's constants against the header, and its refusals that need no GPU."""
import os
import re

from paper_2608_17310_gb300 import rollout as ro

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_constants_are_the_headers():
    with open(os.path.join(ROOT, "include", "es_rollout.h")) as f:
        defined = dict(re.findall(r"#define (ES_\w+) (\d+)", f.read()))
    assert {k: int(v) for k, v in defined.items()} == {k: getattr(ro, k) for k in defined}
    assert {"ES_MAX_SEQUENCES", "ES_ATTENTION_GAVE_UP"} <= set(defined)
