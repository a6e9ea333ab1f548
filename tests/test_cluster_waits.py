"""Barriers that other CTAs' stores complete are waited for with an acquire of the cluster's scope (a wait without a scope acquires the CTA's alone, and
does not order reads behind stores that another CTA made).  Read from the sources: on the device a weaker wait may go right for years."""
import pathlib
import re

import paper_2203_05705_b200

CSRC = pathlib.Path(paper_2203_05705_b200.__file__).parent / "csrc"


def test_the_recurrences_mail():
    text = (CSRC / "glr.cu").read_text()
    waits = re.findall(r"(\w+)\(smem_u32\(&sh\.post\.bar\[[^;]*;", text)
    assert "st.async" in text and waits
    assert {w for w in waits if "wait" in w} == {"mbar_wait_cluster"}


def test_every_kernel_that_stores_into_another_ctas_memory():
    for path in sorted(CSRC.glob("*.cu")):
        text = path.read_text()
        if re.search(r'"[^"]*st\.async', text):
            assert "mbar_wait_cluster(" in text, path.name
    header = (CSRC / "sm100_ptx.h").read_text()
    body = header[header.index("bool mbar_wait_cluster("):]
    assert "acquire.cluster" in body[:body.index("\n}\n")]
