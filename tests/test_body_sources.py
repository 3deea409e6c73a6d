"""Rules of the kernels' sources that no run can show reliably."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_06619_b200", "csrc")


def _functions_that_wait():
    """(file, head, body) of every function that begins before the kernel in front of it has ended."""
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for call in re.finditer(r"^  +wait_for_primary\(\);", text, flags=re.M):
            # functions start in column 0 and end with a closing brace there
            start = text.rfind("\n}", 0, call.start()) + 2
            end = text.index("\n}", call.start())
            head, body = text[start:end].split("{", 1)
            yield name, head, body


def test_data_of_an_overlapped_kernel_is_not_read_through_the_read_only_path():
    found = list(_functions_that_wait())
    assert {f[0] for f in found} >= {"nat_attn_bf16.cu", "nat_attn_bwd_bf16.cu", "nat_resnorm.cu"}
    assert len(found) >= 6
    for name, head, body in found:
        assert "__ldg(" not in body, name
        assert not re.search(r"const\s+\w+\s*\*\s*__restrict__", head), name


def test_every_device_helper_is_reached():
    texts = {n: open(os.path.join(CSRC, n)).read() for n in os.listdir(CSRC)}
    everything = "\n".join(texts.values())
    for name, text in sorted(texts.items()):
        for helper in set(re.findall(r"__forceinline__[^;{}()]*?\b(\w+)\(", text)):
            if helper != "operator":
                uses = re.findall(r"\b%s\b *[(<]" % helper, everything)
                defined = re.findall(r"__forceinline__[^;{}()]*?\b%s\(" % helper, everything)
                assert len(uses) > len(defined), (name, helper)
