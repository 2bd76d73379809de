"""The bench's counter traffic: taken from the committed summaries of the verifier's own kernels, whatever becomes of the
sources that the verifier does not use (CPU)."""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import bench  # noqa: E402
from paper_2608_03447_amd import build  # noqa: E402

HEADLINE = "b256_k16_v151936_bf16"


def test_the_headline_has_its_counter_traffic():
    algorithmic = 4352 * 151936 * 2
    traffic = bench.read_traffic(HEADLINE, bench.kernel_source_hash())
    assert traffic is not None and algorithmic <= traffic < 1.01 * algorithmic
    assert bench.read_traffic(HEADLINE + "_d5120", bench.kernel_source_hash(), "asd_lmhead_kernel") is not None


def test_traffic_of_other_sources_is_not_taken():
    assert bench.read_traffic(HEADLINE, "0123456789abcdef") is None


def test_the_hash_is_of_the_verifier_alone(monkeypatch):
    before = bench.kernel_source_hash()
    monkeypatch.setattr(build, "DECODE_SOURCES", [])
    monkeypatch.setattr(build, "DECODE_HEADERS", [])
    assert bench.kernel_source_hash() == before
