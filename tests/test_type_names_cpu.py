"""One definition of a type for the whole library: its sources share a namespace, so no two of them may give a name to different types."""
import re
from collections import defaultdict
from pathlib import Path

SOURCES = Path(__file__).resolve().parents[1] / "paper_2412_03409_amd" / "csrc"
HEAD = re.compile(r"^(?:template\s*<[^{;]*>\s*)?(?:struct|class|union|enum(?:\s+class)?)\s+(\w+)[^;{]*\{", re.M)


def test_no_two_sources_define_a_type_of_the_same_name():
    where = defaultdict(set)
    for path in sorted((p for p in SOURCES.iterdir() if p.suffix in (".hip", ".hpp"))):
        for name in HEAD.findall(path.read_text()):
            where[name].add(path.name)
    assert len(where) > 30                                      # the pattern still finds them
    assert {n: sorted(f) for n, f in where.items() if len(f) > 1} == {}
