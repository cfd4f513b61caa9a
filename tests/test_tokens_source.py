"""What the sources of the tokens' kernels have to say for themselves, because no run shows it: lanes of a wavefront that exchange values through LDS."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2008_03433_amd", "csrc")
FENCE = "wave_lds_fence();"

# function, and accesses of one place by several lanes in the order of the source: a fence stands between each two that follow each other
EXCHANGES = {
    "head_beam.hip": [
        ("cut_to", [FENCE, "list[i * kWave + lane] : 0", "if (keep) list[", "return bound;"]),
        ("k_beam_offers", [FENCE, "looked[wave][q][", "= looked[wave][lane"]),
        ("k_beam_offers", ["if (in) list[count", "lane < count ? list[lane] : 0;\n        const bool in"]),
        ("k_beam_offers", ["= join[read + i]", "list[count + i] ="]),
    ],
    "head_embed.hip": [
        ("k_sort_tokens", ["mark[k] = ", "mark[k] != lane"]),
        ("k_sort_tokens", ["const int at = counts[wave][token];", "if (lane == 0) counts[wave][token] =", "const int at = counts[wave][k];", "};\n    if (own_here"]),
    ],
}


def _body(text, name):
    """A function's text, to the closing brace in the first column."""
    start = re.search(rf"\b{name}\(", text).start()
    return text[start:text.index("\n}\n", start)]


@pytest.mark.parametrize("file", sorted(EXCHANGES))
def test_exchanges_of_a_wavefront_lie_between_fences(file):
    with open(os.path.join(CSRC, file)) as f:
        text = re.sub(r"[ \t]*//[^\n]*", "", f.read())
    for name, accesses in EXCHANGES[file]:
        body = _body(text, name)
        places = [body.index(a) for a in accesses]
        assert places == sorted(places), (file, accesses)
        for a, b in zip(places, places[1:]):
            assert FENCE in body[a:b], (file, accesses, body[a:b])
