"""The gradient's sort: what its CTAs read of each other's shared memory is written once
between two barriers of the cluster.

A CTA that has passed the barrier after which the others' counts are read may run ahead of
them by a whole tile, so nothing but the exchange itself may write those counts.  Read from
the kernel's source: a CTA that is late enough for it to show cannot be arranged."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def sort_kernel():
    text = open(os.path.join(ROOT, "paper_2607_13093_gb300", "csrc", "k_table.cu")).read()
    text = re.sub(r"//[^\n]*", "", text)
    body = text[text.index("sort_kernel(const TableGrad a"):]
    return body[:body.index("__global__")]


def block(text, at):
    """The braces that open at or after `at`, with what they hold."""
    start = text.index("{", at)
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return start, i + 1
    raise AssertionError("unbalanced braces")


def writes(text, name):
    w = r"\bs\." + name + r"\[[^\]]*\]\s*(?:[-+|&^]?=(?!=)|\+\+|--)"
    atomic = r"atomic\w+\(\s*&\s*s\." + name + r"\["
    return [m.start() for m in re.finditer(f"{w}|{atomic}", text)]


def test_counts_read_by_the_cluster_are_written_by_the_exchange_alone():
    body = sort_kernel()
    remote = set(re.findall(r"mapa\(ptx::smem_u32\(&s\.(\w+)\[", body))
    assert remote
    a, b = block(body, body.index("auto place ="))
    exchange = body[a:b]
    for name in remote:
        at = writes(body, name)
        assert len(at) == 1 and a < at[0] < b, (name, [body[i:i + 40] for i in at])
        # written, then the barrier, then read
        order = [writes(exchange, name)[0], exchange.index("cluster_sync"), exchange.index("mapa")]
        assert order == sorted(order)
    # one exchange a pass (which one depends on the list's length), and a barrier at its end
    calls = [m.start() for m in re.finditer(r"\bplace\(", body)]
    assert len(calls) == 2
    assert re.search(r"if \(!one\)", body) and re.search(r"if \(one && !local\) place\(", body)
    assert body.index("cluster_sync", max(calls)) > max(calls)
