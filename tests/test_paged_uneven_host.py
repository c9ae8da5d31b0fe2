"""What the page kernels rely on, by their sources: alignment of what is read 16 bytes at a time, and words
that a call which fails half-way leaves as the next one wants them."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_14256_b200", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["zc_paged_decode.cu", "zc_paged_chunk.cu", "zc_paged_own.cu", "zc_paged_weights.cu", "zc_page_evict.cu"])
def test_shared_memory_of_bulk_accesses_is_declared_aligned(name):
    """Copies and accesses of 16 bytes: the dynamic shared memory says so itself, whatever static variables lie before it."""
    found = re.findall(r"extern __shared__ ([^;]*);", source(name))
    assert found
    for what in found:
        align = re.search(r"__align__\((\d+)\)", what)
        assert (align and int(align.group(1)) >= 16) or what.startswith("uint4 "), what


def test_a_shared_call_that_fails_half_way_leaves_its_word_clear():
    """The first of the three kernels sets a word that the last one clears.  Whatever can fail beside the launches comes
    before the first of them, and a failed launch behind it clears the word on the stream."""
    text = source("zc_paged_chunk.cu")
    body = text[text.index("int zc_launch_paged_shared("):]
    body = body[:body.index("\n}\n")]
    ask, first = body.index("logits, false, st)"), body.index("launch_groups<__half>")
    rest, clear = body.index("logits, true, st)"), body.index("cudaMemsetAsync(k.gr.told, 0, sizeof(int), st)")
    assert body.index("make_q_map(") < ask < first < rest < clear
    assert all(body.index(x) < first for x in ("zc_page_maps(", "return (int)cudaErrorNotSupported"))
    assert re.search(r"if \(e != cudaSuccess\) return e;", body[ask:first]) and re.search(r"if \(e != cudaSuccess\) $", body[:clear])
    assert "return" not in body[rest:clear]
    own = source("zc_paged_own.cu")
    launch = own[own.index("cudaError_t launch("):own.index("cudaError_t launch_mode(")]
    assert launch.index("zc_allow_smem(") < launch.index("|| !go) return e;") < launch.index("zc_launch_early(")
    end = own[own.index("int zc_launch_own_keys("):]
    assert end.index("|| !go) return") < end.index("launch_join_rows<") and "zc_allow_smem" not in end
    # nobody else clears or sets it
    assert own.count("*k.gr.told = 0") == 1 and text.count("k.gr.told") == 2
