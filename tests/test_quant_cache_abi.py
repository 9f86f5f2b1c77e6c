"""The binding's structures of the 8-bit cache and of the rotation with several axes are the header's; their entry points refuse a
missing context without a GPU."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_binding_structs_of_the_8_bit_cache_match_the_header():
    from paper_2511_13587_b200 import binding as vb
    text = open(os.path.join(ROOT, "include", "vvs.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for struct in (vb.vvs_heads, vb.vvs_rope_axes, vb.vvs_qcache):
        body = re.search(r"typedef struct %s \{(.*?)\}" % struct.__name__, text, flags=re.S).group(1)
        assert re.findall(r"(\w+)\s*;", body) == [f[0] for f in struct._fields_], struct.__name__
    assert vb.lib.vvs_rotate_axes(None, None, 1, 1, 1, 1, 64, None, None, None, None, None) == -1
    assert vb.lib.vvs_quant_cache_append(None, None, None, None, None, 1, None, None, None, None, 0, None, None, None) == -1
    assert vb.lib.vvs_quant_cache_attend(None, None, None, None, None, 1, 1, None, None, None, None, 0.0, 0, 1.0, 0, None) == -1
    assert vb.lib.vvs_quant_cache_evict(None, None, None, 1, 0, 0, None, None, None, None, None, None) == -1
    assert vb.lib.vvs_element_bytes(None) == -1
